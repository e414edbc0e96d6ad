// Rows of features: their three types, and the checks that the calls on rows share.
#pragma once

#include "nd_common.h"

namespace nd {

using bf16_t = __bf16;
using f16_t = _Float16;

// 16 bytes of a row (or one number), at any address: the memory takes wide loads and stores wherever they lie.
template <typename T, int N>
struct Piece {
    T v[N];
};
template <typename T, int N>
__device__ __forceinline__ Piece<T, N> load_piece(const T* from) {
    Piece<T, N> p;
    __builtin_memcpy(&p, from, sizeof(p));
    return p;
}
template <typename T, int N>
__device__ __forceinline__ void store_piece(T* to, const Piece<T, N>& p) {
    __builtin_memcpy(to, &p, sizeof(p));
}

inline size_t dtype_bytes(int dtype) { return dtype == ND_F32 ? 4 : 2; }

// What every call on rows refuses.  n rows of d numbers, `stride` apart.
inline int check_rows(const char* what, const void* rows, int64_t n, int32_t d, int64_t stride, int dtype) {
    if (n > 0 && !rows) {
        set_error("%s is NULL", what);
        return ND_ERR_NULL_POINTER;
    }
    if (stride < d) {
        set_error("%s: rows of %d numbers cannot lie %lld apart", what, d, (long long)stride);
        return ND_ERR_BAD_ARGUMENT;
    }
    // what a kernel adds to the address has to fit in 63 bits
    if (n > 0 && stride > (int64_t)(1ll << 62) / n / 4) {
        set_error("%s: %lld rows %lld numbers apart", what, (long long)n, (long long)stride);
        return ND_ERR_TOO_LARGE;
    }
    if (((uintptr_t)rows % dtype_bytes(dtype)) != 0) {
        set_error("%s is not aligned to its type", what);
        return ND_ERR_BAD_ARGUMENT;
    }
    return ND_OK;
}
inline int check_row_type(int dtype, int32_t d) {
    if (dtype != ND_F32 && dtype != ND_BF16 && dtype != ND_F16) {
        set_error("dtype %d is none of nd_dtype", dtype);
        return ND_ERR_BAD_ARGUMENT;
    }
    if (d < 1 || d > ND_MAX_ROW) {
        set_error("rows have %d numbers; 1 to %d", d, ND_MAX_ROW);
        return d < 1 ? ND_ERR_BAD_ARGUMENT : ND_ERR_TOO_LARGE;
    }
    return ND_OK;
}

}  // namespace nd
