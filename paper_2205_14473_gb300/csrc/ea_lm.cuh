// ea_lm.cuh -- what the units of include/ea_lm.h share: element types, launches, the list of gradients that a
// launch carries, and the host's checks.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <new>
#include <utility>
#include <vector>

#include "ea_internal.h"
#include "ea_lm.h"

namespace ea {

using bf16 = __nv_bfloat16;
using f16 = __half;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(f16 x) { return __half2float(x); }

template <class T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ f16 from_f32<f16>(float x) { return __float2half_rn(x); }

// Two binary32 values in one 64-bit register: one instruction slot for two operations, each rounded by itself.
struct F2 {
    unsigned long long v;
};
__device__ __forceinline__ F2 pack2(float a, float b)
{
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(F2 x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ F2 add2(F2 a, F2 b)
{
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c)
{
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ F2 times2(F2 a, F2 b)
{
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 both(float a) { return pack2(a, a); }

inline size_t type_bytes(int32_t type) { return type == EA_T_F32 || type == EA_T_I32 ? 4 : type == EA_T_I64 ? 8 : 2; }
inline bool is_float_type(int32_t type) { return type == EA_T_F32 || type == EA_T_BF16 || type == EA_T_F16; }

// A failure without a handle of ea.h: the text goes to ea_last_error(NULL).
inline int lm_fail(int code, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        set_last_error(buf);
    } catch (const std::bad_alloc &) {
    }
    return code;
}

inline int lm_cuda(cudaError_t e, const char *what)
{
    return e == cudaSuccess ? EA_OK : lm_fail(EA_E_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

inline int check_workspace(const void *p, size_t have, size_t need)
{
    if (!p) return lm_fail(EA_E_WORKSPACE, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(p) % 256) return lm_fail(EA_E_WORKSPACE, "workspace is not 256-byte aligned");
    if (have < need) return lm_fail(EA_E_WORKSPACE, "workspace has %zu bytes, needs %zu", have, need);
    return EA_OK;
}

inline int check_address(const void *p, int32_t type, const char *what)
{
    if (!p) return lm_fail(EA_E_INVAL, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(p) % type_bytes(type))
        return lm_fail(EA_E_ALIGN, "%s is not aligned to its %zu-byte elements", what, type_bytes(type));
    return EA_OK;
}

// The device that is current at a handle's init call, and its SMs.
struct DeviceOf {
    int id = 0, sms = 0;
    int query()
    {
        const int r = lm_cuda(cudaGetDevice(&id), "current device");
        return r != EA_OK ? r : lm_cuda(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, id), "SM count");
    }
    int check() const
    {
        int now = -1;
        const int r = lm_cuda(cudaGetDevice(&now), "current device");
        if (r != EA_OK) return r;
        return now == id ? EA_OK : lm_fail(EA_E_INVAL, "the handle belongs to device %d, device %d is current", id, now);
    }
};

// SMs that a workspace is sized for (a handle uses no more of them).
constexpr int kMaxSms = 160;

// Launch `kernel` in clusters of `cluster` CTAs; with `overlap`, it may begin before its predecessor has finished
// (programmatic dependent launch; see pdl_wait).
template <class... KArgs, class... Args>
cudaError_t launch_lm(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, cudaStream_t s, bool overlap, int cluster, Args &&...args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(block));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    unsigned n = 0;
    if (overlap) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = static_cast<unsigned>(cluster);
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

// Tensors whose gradients one launch carries as a parameter.
constexpr int kGradBatch = 448;
struct GradList {
    const void *g[kGradBatch];
};

// Groups of cp.async: the copies issued since the last commit are one; wait until all but the last N are done.
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// The tensor of unit u: the last one whose first unit is <= u (empty tensors have none).  hint: one whose first
// unit is <= u.
__device__ __forceinline__ int tensor_of(const int64_t *first, int n, int64_t u, int hint)
{
    int lo = hint, hi = n - 1;
    if (u < first[lo + 1]) return lo;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

}  // namespace ea
