// ea_block.cuh -- what the units of include/ea_block.h share: rows of a batch, accesses, checks.
#pragma once

#include <type_traits>

#include "ea_block.h"
#include "ea_lm.cuh"

namespace ea {

constexpr int64_t kMaxRows = int64_t{1} << 30;

// Row r of a call is row (i, j) of the batch, i = r / inner.  The division of r < 2^30 by the constant inner >= 2 is a
// multiplication (Granlund and Montgomery, "Division by invariant integers using multiplication"): with
// s = ceil(log2 inner) and magic = floor(2^(31 + s) / inner) + 1 < 2^32 the error stays below 1 / inner.
struct Rows {
    uint32_t inner = 0, magic = 0;  // inner = 0: all rows are in one row of the batch
    int shift = 0;

    __device__ __forceinline__ uint32_t outer_of(uint32_t r) const { return inner ? __umulhi(r, magic) >> shift : 0; }
};

inline Rows rows_of(int64_t inner)
{
    Rows r;
    int s = 0;
    while ((int64_t{1} << s) < inner) ++s;
    r.inner = static_cast<uint32_t>(inner);
    r.magic = static_cast<uint32_t>((uint64_t{1} << (31 + s)) / inner + 1);
    r.shift = s - 1;
    return r;
}

// A tensor of rows: element 0 of row (i, j) at p + i * outer + j * inner.
template <class T>
struct RowsOf {
    T *p;
    int64_t outer, inner;

    __device__ __forceinline__ T *row(const Rows &rows, uint32_t r) const
    {
        const uint32_t i = rows.outer_of(r);
        return p + (i * outer + static_cast<int64_t>(r - i * rows.inner) * inner);
    }
};

// A value of a runtime type.
__device__ __forceinline__ float load_any(const void *p, int32_t type, int64_t i)
{
    return type == EA_T_F32    ? static_cast<const float *>(p)[i]
           : type == EA_T_BF16 ? to_f32(static_cast<const bf16 *>(p)[i])
                               : to_f32(static_cast<const f16 *>(p)[i]);
}
__device__ __forceinline__ void store_any(void *p, int32_t type, int64_t i, float x)
{
    if (type == EA_T_F32) static_cast<float *>(p)[i] = x;
    else if (type == EA_T_BF16) static_cast<bf16 *>(p)[i] = from_f32<bf16>(x);
    else static_cast<f16 *>(p)[i] = from_f32<f16>(x);
}

__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = __fadd_rn(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}

template <class T>
constexpr T over(T a, T b) { return (a + b - 1) / b; }
constexpr size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// f(a pointer of the element type) for the type at hand.
template <class F>
void with_float(int32_t type, F f)
{
    switch (type) {
    case EA_T_F32: f(static_cast<float *>(nullptr)); break;
    case EA_T_BF16: f(static_cast<bf16 *>(nullptr)); break;
    default: f(static_cast<f16 *>(nullptr));
    }
}

// f(x, y) for a pair of the same types, or with x (y, where `either`) binary32 and the other one of 16 bits.
template <class F>
void with_pair(int32_t x, int32_t y, F f)
{
    with_float(x, [&](auto *a) {
        with_float(y, [&](auto *b) {
            using A = std::remove_reference_t<decltype(*a)>;
            using B = std::remove_reference_t<decltype(*b)>;
            if constexpr (std::is_same<A, B>::value || std::is_same<A, float>::value || std::is_same<B, float>::value) f(a, b);
        });
    });
}

// Rows of `dim` elements that are written: apart from one another.
inline int check_rows_apart(int64_t outer, int64_t inner, int64_t outer_stride, int64_t inner_stride, int64_t dim, const char *what)
{
    if (!outer || !inner) return EA_OK;
    int64_t n[2] = {inner, outer}, s[2] = {inner_stride, outer_stride};
    if (n[1] > 1 && (n[0] <= 1 || s[1] < s[0])) std::swap(n[0], n[1]), std::swap(s[0], s[1]);
    const bool small = n[0] <= 1 || s[0] >= dim;
    const bool large = n[1] <= 1 || (small && s[1] >= dim && (s[1] - dim) / s[0] >= n[0] - 1);
    return small && large ? EA_OK : lm_fail(EA_E_INVAL, "the rows of %s overlap", what);
}

// The kernels of a handle that may have more shared memory than the 48 KB, their own variables included, that they get unasked, or
// clusters of 16: asked for once each.
struct Allowed {
    const void *kernels[16] = {};
    template <class K>
    cudaError_t operator()(K *kernel, size_t bytes, bool large_cluster = false)
    {
        const void *k = reinterpret_cast<const void *>(kernel);
        const size_t at = reinterpret_cast<uintptr_t>(k) / 16 % 16;
        if (kernels[at] == k || (bytes <= 16 * 1024 && !large_cluster)) return cudaSuccess;
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
        if (e == cudaSuccess && large_cluster) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e == cudaSuccess) kernels[at] = k;
        return e;
    }
};

// Whether every row of a tensor starts on a boundary of `bytes` and is whole vectors of it.
inline bool rows_on(size_t bytes, const void *p, int32_t type, int64_t dim, int64_t outer, int64_t inner, int64_t outer_stride, int64_t inner_stride)
{
    const int64_t vec = static_cast<int64_t>(bytes / type_bytes(type));
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && dim % vec == 0 && (outer <= 1 || outer_stride % vec == 0) &&
           (inner <= 1 || inner_stride % vec == 0);
}

}  // namespace ea
