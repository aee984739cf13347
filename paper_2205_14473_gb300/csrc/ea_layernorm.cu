// ea_layernorm.cu -- ea_layernorm_forward and ea_layernorm_backward.
//
// Both are one pass over the rows.  A group of lanes or warps holds a row in registers, 16 elements a thread, and the next row's
// loads are on their way while it works on this one.  Mean and variance: each warp's mean and the squares about it, joined
// (Chan, Golub and LeVeque, "Updating formulae and a pairwise algorithm for computing sample variances"), so that the variance
// does not cancel and a row costs one barrier.  The gradients of weight and bias are sums over rows: every thread keeps
// those of its columns, a CTA's groups are added at its end, and a second launch adds the CTAs' in order.
// Rows that registers do not hold are read from the caches again.
#include "ea_async.cuh"
#include "ea_block.cuh"

namespace ea {

constexpr int kNormRowThreads = 256;
constexpr int kColumnLanes = 32, kColumnRows = 8;  // a CTA of the column sums: columns, and rows at a time

struct LnArgs {
    uint32_t n;         // rows
    Rows rows;
    int64_t dim;
    float eps, inverse; // inverse: 1 / dim
    const void *w, *b;
    int32_t weight_type, grad_type;
};

// The CTA's sum in every thread.
__device__ __forceinline__ float row_block_sum(float v, float *red)
{
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kNormRowThreads / 32; ++i) s = __fadd_rn(s, red[i]);
    return s;
}

// Any width: a CTA takes a row, and reads it three times (the first time from memory).
template <class X, class Y>
__global__ void __launch_bounds__(kNormRowThreads) ln_forward_any_kernel(const LnArgs a, const RowsOf<const X> xs, const RowsOf<Y> ys, float *stats)
{
    __shared__ float red[kNormRowThreads / 32];
    for (uint32_t r = blockIdx.x; r < a.n; r += gridDim.x) {
        const X *x = xs.row(a.rows, r);
        Y *y = ys.row(a.rows, r);
        float s = 0.0f;
        for (int64_t i = threadIdx.x; i < a.dim; i += kNormRowThreads) s = __fadd_rn(s, to_f32(x[i]));
        const float mean = __fmul_rn(row_block_sum(s, red), a.inverse);
        s = 0.0f;
        for (int64_t i = threadIdx.x; i < a.dim; i += kNormRowThreads) {
            const float d = __fsub_rn(to_f32(x[i]), mean);
            s = __fmaf_rn(d, d, s);
        }
        const float rstd = __frsqrt_rn(__fmaf_rn(row_block_sum(s, red), a.inverse, a.eps));
        for (int64_t i = threadIdx.x; i < a.dim; i += kNormRowThreads) {
            float t = __fmul_rn(__fsub_rn(to_f32(x[i]), mean), rstd);
            if (a.w) t = __fmul_rn(t, load_any(a.w, a.weight_type, i));
            if (a.b) t = __fadd_rn(t, load_any(a.b, a.weight_type, i));
            y[i] = from_f32<Y>(t);
        }
        if (stats && threadIdx.x == 0) *reinterpret_cast<float2 *>(stats + 2 * static_cast<int64_t>(r)) = make_float2(mean, rstd);
    }
}

template <class X, class Y>
__global__ void __launch_bounds__(kNormRowThreads) ln_dx_any_kernel(const LnArgs a, const RowsOf<const Y> dys, const RowsOf<const X> xs, const float *stats,
                                                                    const RowsOf<const X> adds, const RowsOf<X> dxs)
{
    __shared__ float red[kNormRowThreads / 32];
    for (uint32_t r = blockIdx.x; r < a.n; r += gridDim.x) {
        const X *x = xs.row(a.rows, r), *add = adds.p ? adds.row(a.rows, r) : nullptr;
        const Y *dy = dys.row(a.rows, r);
        X *dx = dxs.row(a.rows, r);
        const float2 st = *reinterpret_cast<const float2 *>(stats + 2 * static_cast<int64_t>(r));
        float s = 0.0f, p = 0.0f;
        for (int64_t i = threadIdx.x; i < a.dim; i += kNormRowThreads) {
            float q = to_f32(dy[i]);
            if (a.w) q = __fmul_rn(q, load_any(a.w, a.weight_type, i));
            s = __fadd_rn(s, q);
            p = __fmaf_rn(q, __fmul_rn(__fsub_rn(to_f32(x[i]), st.x), st.y), p);
        }
        s = __fmul_rn(row_block_sum(s, red), a.inverse);
        p = __fmul_rn(row_block_sum(p, red), a.inverse);
        for (int64_t i = threadIdx.x; i < a.dim; i += kNormRowThreads) {
            float q = to_f32(dy[i]);
            if (a.w) q = __fmul_rn(q, load_any(a.w, a.weight_type, i));
            const float t = __fmul_rn(__fsub_rn(to_f32(x[i]), st.x), st.y);
            const float d = __fmul_rn(st.y, __fmaf_rn(-t, p, __fsub_rn(q, s)));
            dx[i] = from_f32<X>(add ? __fadd_rn(d, to_f32(add[i])) : d);
        }
    }
}

// Sums of a tile of 32 columns over the rows of one part of the call, into partial[part]: dw's dim values, then db's.
template <class X, class Y>
__global__ void __launch_bounds__(kColumnLanes *kColumnRows) ln_columns_any_kernel(const LnArgs a, const RowsOf<const Y> dys, const RowsOf<const X> xs,
                                                                                   const float *stats, uint32_t part_rows, float *partial)
{
    __shared__ float red[2][kColumnRows][kColumnLanes];
    const int64_t column = static_cast<int64_t>(blockIdx.x) * kColumnLanes + threadIdx.x;
    const uint32_t first = blockIdx.y * part_rows, last = min(a.n, first + part_rows);
    float w = 0.0f, b = 0.0f;
    if (column < a.dim)
        for (uint32_t r = first + threadIdx.y; r < last; r += kColumnRows) {
            const float2 st = *reinterpret_cast<const float2 *>(stats + 2 * static_cast<int64_t>(r));
            const float dy = to_f32(dys.row(a.rows, r)[column]);
            w = __fmaf_rn(dy, __fmul_rn(__fsub_rn(to_f32(xs.row(a.rows, r)[column]), st.x), st.y), w);
            b = __fadd_rn(b, dy);
        }
    red[0][threadIdx.y][threadIdx.x] = w;
    red[1][threadIdx.y][threadIdx.x] = b;
    __syncthreads();
    if (threadIdx.y < 2 && column < a.dim) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kColumnRows; ++i) s = __fadd_rn(s, red[threadIdx.y][i][threadIdx.x]);
        partial[(static_cast<int64_t>(blockIdx.y) * 2 + threadIdx.y) * a.dim + column] = s;
    }
}

// The parts' sums added in order: a CTA takes 32 columns of dw (blockIdx.y = 0) or db.
__global__ void __launch_bounds__(kColumnLanes *kColumnRows) ln_join_kernel(const LnArgs a, const float *partial, int parts, void *dw, void *db, int accumulate)
{
    __shared__ float red[kColumnRows][kColumnLanes];
    const int lane = threadIdx.x % kColumnLanes, row = threadIdx.x / kColumnLanes;
    void *out = blockIdx.y ? db : dw;
    pdl_wait();
    if (!out) return;
    const int64_t column = static_cast<int64_t>(blockIdx.x) * kColumnLanes + lane;
    float s = 0.0f;
    if (column < a.dim)
#pragma unroll 4
        for (int k = row; k < parts; k += kColumnRows) s = __fadd_rn(s, partial[(static_cast<int64_t>(k) * 2 + blockIdx.y) * a.dim + column]);
    red[row][lane] = s;
    __syncthreads();
    if (row || column >= a.dim) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < kColumnRows; ++i) s = __fadd_rn(s, red[i][lane]);
    if (accumulate) s = __fadd_rn(s, load_any(out, a.grad_type, column));
    store_any(out, a.grad_type, column, s);
}

// ---------------------------------------------------------------------------------------------- rows in registers
constexpr int kHeld = 16;                // elements of a thread
constexpr int kBackThreads = 512;
constexpr int kForwardDepth = 4;         // rows on their way
// Of the gradient: what 192 KB hold of x, dy and the added rows.
template <class X, class Y>
constexpr int kBackDepth = 192 * 1024 / (kBackThreads * kHeld * (2 * static_cast<int>(sizeof(X)) + static_cast<int>(sizeof(Y))));

// An 8-byte asynchronous copy global -> shared.
__device__ __forceinline__ void cp_async8(void *dst, const void *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_addr(dst)), "l"(src) : "memory");
}

// A thread's 16 elements of a row: packs of VEC, pack k of lane l of a group of G being pack l + k G of the row.
template <class T, int VEC>
struct Held {
    struct alignas(VEC * sizeof(T)) Pack {
        T x[VEC];
    };
    static constexpr int kPacks = kHeld / VEC;
    Pack p[kPacks];

    // Packs k of a row on their way to `slots` (one of them to every kStep-th), none of those outside the row.
    template <int G, int kStep>
    static __device__ __forceinline__ void fetch(Pack *slots, const T *row, int lane, int packs)
    {
#pragma unroll
        for (int k = 0; k < kPacks; ++k)
            if (lane + k * G < packs) {
                if constexpr (sizeof(Pack) == 16) cp_async16(slots + k * kStep, row + (lane + k * G) * VEC);
                else cp_async8(slots + k * kStep, row + (lane + k * G) * VEC);
            }
    }
    template <int kStep>
    static __device__ __forceinline__ void clear(Pack *slots)
    {
#pragma unroll
        for (int k = 0; k < kPacks; ++k) slots[k * kStep] = Pack{};
    }
    template <int kStep>
    __device__ __forceinline__ void take(const Pack *slots)
    {
#pragma unroll
        for (int k = 0; k < kPacks; ++k) p[k] = slots[k * kStep];
    }
    template <int G>
    __device__ __forceinline__ void load(const T *row, int lane, int packs)
    {
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const int i = lane + k * G;
            if (i < packs) p[k] = reinterpret_cast<const Pack *>(row)[i];
            else p[k] = Pack{};
        }
    }
    __device__ __forceinline__ void values(F2 (&y)[kHeld / 2]) const
    {
#pragma unroll
        for (int i = 0; i < kHeld / 2; ++i) {
            const int k = 2 * i / VEC, j = 2 * i % VEC;
            if constexpr (std::is_same<T, bf16>::value && VEC > 1) {
                const uint32_t w = *reinterpret_cast<const uint32_t *>(p[k].x + j);
                y[i] = pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
            } else if constexpr (std::is_same<T, f16>::value && VEC > 1) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(p[k].x + j));
                y[i] = pack2(f.x, f.y);
            } else if constexpr (VEC > 1) {
                y[i] = pack2(to_f32(p[k].x[j]), to_f32(p[k].x[j + 1]));
            } else {
                y[i] = pack2(to_f32(p[2 * i].x[0]), to_f32(p[2 * i + 1].x[0]));
            }
        }
    }
    template <int G>
    static __device__ __forceinline__ void store(T *row, int lane, int packs, const F2 (&y)[kHeld / 2])
    {
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            Pack q;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int i = k * VEC + j;
                float a, b;
                unpack2(y[i / 2], a, b);
                q.x[j] = from_f32<T>(i & 1 ? b : a);
            }
            if (lane + k * G < packs) reinterpret_cast<Pack *>(row)[lane + k * G] = q;
        }
    }
};

// The same elements of a weight of any type and alignment; `fill` for a weight that is NULL and outside the row.
template <int VEC, int G>
__device__ __forceinline__ void load_weight(const void *w, int32_t type, int lane, int packs, float fill, F2 (&y)[kHeld / 2])
{
    float f[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int pack = lane + i / VEC * G;
        f[i] = w && pack < packs ? load_any(w, type, static_cast<int64_t>(pack) * VEC + i % VEC) : fill;
    }
#pragma unroll
    for (int i = 0; i < kHeld / 2; ++i) y[i] = pack2(f[2 * i], f[2 * i + 1]);
}

__device__ __forceinline__ F2 times2(F2 a, F2 b)
{
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ float total(F2 a)
{
    float x, y;
    unpack2(a, x, y);
    return __fadd_rn(x, y);
}
template <int G>
__device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1) x = __fadd_rn(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
// A barrier of the G threads of a group (G a multiple of 32).
template <int G>
__device__ __forceinline__ void group_sync(int group)
{
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(G) : "memory");
}

// A CTA is a group of warps, or 128 threads of smaller groups.
template <class X, class Y, int VEC, int G>
__global__ void __launch_bounds__(G > 32 ? G : 128) ln_forward_kernel(const LnArgs a, const RowsOf<const X> xs, const RowsOf<Y> ys, float *stats)
{
    constexpr int kThreads = G > 32 ? G : 128, kGroups = kThreads / G, W = G / 32, kDepth = kForwardDepth;
    constexpr bool kRing = VEC > 1;
    using H = Held<X, VEC>;
    using Pack = typename H::Pack;
    extern __shared__ __align__(16) unsigned char memory[];
    Pack *ring = reinterpret_cast<Pack *>(memory) + threadIdx.x;  // a stage: kPacks, one per thread each
    __shared__ float2 parts[2][W > 1 ? W : 1];  // each warp's mean and squares about it, of this row and the last
    __shared__ float share[W > 1 ? W : 1], counts[W > 1 ? W : 1];  // each warp's elements, and their share of the row's
    const int lane = threadIdx.x % G, packs = static_cast<int>(a.dim / VEC), warp = threadIdx.x / 32;
    const uint32_t stride = gridDim.x * kGroups;
    uint32_t r = blockIdx.x * kGroups + threadIdx.x / G;
    F2 w[kHeld / 2], b[kHeld / 2];
    H next;
    auto fetch = [&](uint32_t row, int stage) {
        if constexpr (kRing) {
            if (row < a.n) H::template fetch<G, kThreads>(ring + stage * (H::kPacks * kThreads), xs.row(a.rows, row), lane, packs);
            cp_async_commit();
        } else {
            next.template load<G>(xs.row(a.rows, row), lane, row < a.n ? packs : 0);
        }
    };
    if constexpr (kRing)
        for (int d = 0; d < kDepth; ++d) H::template clear<kThreads>(ring + d * (H::kPacks * kThreads));
    for (int d = 0; d < (kRing ? kDepth : 1); ++d) fetch(r + d * stride, d);
    int stage = 0;
    load_weight<VEC, G>(a.w, a.weight_type, lane, packs, 1.0f, w);
    load_weight<VEC, G>(a.b, a.weight_type, lane, packs, 0.0f, b);
    // elements of this thread's warp (or group), of the packs that lie inside the row
    auto count_of = [&](int first) {
        int n = 0;
#pragma unroll
        for (int k = 0; k < kHeld / VEC; ++k) n += min(max(packs - (first + k * G), 0), G < 32 ? G : 32);
        return n * VEC;
    };
    const int count = count_of(W > 1 ? warp * 32 : 0);
    const float inverse = count ? __fdiv_rn(1.0f, static_cast<float>(count)) : 0.0f;
    if (W > 1 && threadIdx.x % 32 == 0) {
        counts[warp] = static_cast<float>(count);
        share[warp] = __fdiv_rn(static_cast<float>(count), static_cast<float>(a.dim));
    }
    int buffer = 0;
    // whole warps go on until all of their rows are done
    for (uint32_t first = r - (G < 32 ? threadIdx.x % 32 / G : 0); first < a.n; first += stride, r += stride, buffer ^= 1) {
        F2 x[kHeld / 2];
        if constexpr (kRing) {
            cp_async_wait<kDepth - 1>();
            next.template take<kThreads>(ring + stage * (H::kPacks * kThreads));
        }
        next.values(x);
        fetch(r + (kRing ? kDepth : 1) * stride, stage);
        stage = stage + 1 == kDepth ? 0 : stage + 1;
        F2 s = x[0];
#pragma unroll
        for (int i = 1; i < kHeld / 2; ++i) s = add2(s, x[i]);
        float mean = __fmul_rn(lanes_sum<G>(total(s)), inverse);
        F2 minus = both(-mean), q = both(0.0f);
#pragma unroll
        for (int k = 0; k < kHeld / VEC; ++k)
            if (lane + k * G < packs) {
                if constexpr (VEC > 1) {
#pragma unroll
                    for (int i = k * VEC / 2; i < (k + 1) * VEC / 2; ++i) {
                        const F2 d = add2(x[i], minus);
                        q = fma2(d, d, q);
                    }
                } else {
                    float e, f, g, h;
                    unpack2(x[k / 2], e, f);
                    unpack2(q, g, h);
                    const float d = __fsub_rn(k & 1 ? f : e, mean);
                    q = pack2(__fmaf_rn(d, d, g), h);
                }
            }
        float squares = lanes_sum<G>(total(q));
        if constexpr (W > 1) {
            if (threadIdx.x % 32 == 0) parts[buffer][warp] = make_float2(mean, squares);
            __syncthreads();
            mean = squares = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) mean = __fmaf_rn(share[i], parts[buffer][i].x, mean);
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float2 p = parts[buffer][i];
                const float d = __fsub_rn(p.x, mean);
                squares = __fadd_rn(squares, __fmaf_rn(__fmul_rn(d, d), counts[i], p.y));
            }
            minus = both(-mean);
        }
        const float rstd = __frsqrt_rn(__fmaf_rn(squares, a.inverse, a.eps));
        const F2 scale = both(rstd);
#pragma unroll
        for (int i = 0; i < kHeld / 2; ++i) x[i] = fma2(times2(add2(x[i], minus), scale), w[i], b[i]);
        if (r < a.n) {
            Held<Y, VEC>::template store<G>(ys.row(a.rows, r), lane, packs, x);
            if (stats && lane == 0) *reinterpret_cast<float2 *>(stats + 2 * static_cast<int64_t>(r)) = make_float2(mean, rstd);
        }
    }
}

// One CTA to an SM; groups of G threads walk through the rows, and leave the CTA's sums of dw and db in its part.
template <class X, class Y, int VEC, int G>
__global__ void __launch_bounds__(kBackThreads, 1) ln_backward_kernel(const LnArgs a, const RowsOf<const Y> dys, const RowsOf<const X> xs, const float *stats,
                                                                      const RowsOf<const X> adds, const RowsOf<X> dxs, float *partial)
{
    constexpr int kGroups = kBackThreads / G, W = G / 32, T = kBackThreads, kDepth = kBackDepth<X, Y>;
    constexpr bool kRing = VEC > 1;
    using HX = Held<X, VEC>;
    using HY = Held<Y, VEC>;
    extern __shared__ __align__(16) unsigned char memory[];
    float *sums = reinterpret_cast<float *>(memory);  // at the end: each group's dw, then its db
    // A stage: packs of x, of dy and of the added rows, one per thread each.
    typename HX::Pack *ring_x = reinterpret_cast<typename HX::Pack *>(memory) + threadIdx.x, *ring_add = ring_x + kDepth * HX::kPacks * T;
    typename HY::Pack *ring_y = reinterpret_cast<typename HY::Pack *>(memory + 2 * sizeof(X) * kHeld * T * kDepth) + threadIdx.x;
    __shared__ float2 parts[2][kBackThreads / 32];
    const int lane = threadIdx.x % G, group = threadIdx.x / G, packs = static_cast<int>(a.dim / VEC), warp = threadIdx.x / 32;
    const uint32_t stride = gridDim.x * kGroups;
    uint32_t r = blockIdx.x * kGroups + group;
    F2 w[kHeld / 2], dw[kHeld / 2], db[kHeld / 2];
    HX nx, na;
    HY ny;
    float2 st[kRing ? kDepth : 1];  // of the rows on their way
    auto fetch = [&](uint32_t row, int stage, float2 &s) {  // zeros where there is no such row
        s = row < a.n ? *reinterpret_cast<const float2 *>(stats + 2 * static_cast<int64_t>(row)) : make_float2(0.0f, 0.0f);
        if constexpr (kRing) {
            if (row < a.n) {
                HX::template fetch<G, T>(ring_x + stage * (HX::kPacks * T), xs.row(a.rows, row), lane, packs);
                HY::template fetch<G, T>(ring_y + stage * (HY::kPacks * T), dys.row(a.rows, row), lane, packs);
                if (adds.p) HX::template fetch<G, T>(ring_add + stage * (HX::kPacks * T), adds.row(a.rows, row), lane, packs);
            } else {
                HX::template clear<T>(ring_x + stage * (HX::kPacks * T));
                HY::template clear<T>(ring_y + stage * (HY::kPacks * T));
            }
            cp_async_commit();
        } else {
            const int there = row < a.n ? packs : 0;
            nx.template load<G>(xs.row(a.rows, row), lane, there);
            ny.template load<G>(dys.row(a.rows, row), lane, there);
        }
    };
    if constexpr (kRing)
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            HX::template clear<T>(ring_x + d * (HX::kPacks * T));
            HY::template clear<T>(ring_y + d * (HY::kPacks * T));
            HX::template clear<T>(ring_add + d * (HX::kPacks * T));
            fetch(r + d * stride, d, st[d]);
        }
    load_weight<VEC, G>(a.w, a.weight_type, lane, packs, 1.0f, w);
#pragma unroll
    for (int i = 0; i < kHeld / 2; ++i) dw[i] = db[i] = both(0.0f);
    int buffer = 0, stage = 0;
    for (uint32_t first = r - (G < 32 ? threadIdx.x % 32 / G : 0); first < a.n; first += stride, r += stride, buffer ^= 1) {
        const bool on = r < a.n;
        F2 t[kHeld / 2], q[kHeld / 2];
        if constexpr (kRing) {
            cp_async_wait<kDepth - 1>();
            nx.template take<T>(ring_x + stage * (HX::kPacks * T));
            ny.template take<T>(ring_y + stage * (HY::kPacks * T));
        } else {
            fetch(r, 0, st[0]);
        }
        const F2 minus = both(-st[0].x), scale = both(st[0].y);
        nx.values(t);
        ny.values(q);
#pragma unroll
        for (int i = 0; i < kHeld / 2; ++i) {
            t[i] = times2(add2(t[i], minus), scale);
            dw[i] = fma2(q[i], t[i], dw[i]);
            db[i] = add2(db[i], q[i]);
            q[i] = times2(q[i], w[i]);
        }
        if (adds.p) {
            if constexpr (kRing) na.template take<T>(ring_add + stage * (HX::kPacks * T));
            else na.template load<G>(adds.row(a.rows, r), lane, on ? packs : 0);
        }
        if constexpr (kRing) {
#pragma unroll
            for (int d = 0; d + 1 < kDepth; ++d) st[d] = st[d + 1];
            fetch(r + kDepth * stride, stage, st[kDepth - 1]);
            stage = stage + 1 == kDepth ? 0 : stage + 1;
        }
        if (!dxs.p) continue;
        F2 s2 = q[0], p2 = times2(q[0], t[0]);
#pragma unroll
        for (int i = 1; i < kHeld / 2; ++i) s2 = add2(s2, q[i]), p2 = fma2(q[i], t[i], p2);
        float s = lanes_sum<G>(total(s2)), p = lanes_sum<G>(total(p2));
        if constexpr (W > 1) {
            if (threadIdx.x % 32 == 0) parts[buffer][warp] = make_float2(s, p);
            group_sync<G>(group);
            s = p = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float2 o = parts[buffer][group * W + i];
                s = __fadd_rn(s, o.x);
                p = __fadd_rn(p, o.y);
            }
        }
        const F2 minus_s = both(-__fmul_rn(s, a.inverse)), minus_p = both(-__fmul_rn(p, a.inverse));
#pragma unroll
        for (int i = 0; i < kHeld / 2; ++i) t[i] = times2(fma2(t[i], minus_p, add2(q[i], minus_s)), scale);
        if (adds.p) {
            na.values(q);
#pragma unroll
            for (int i = 0; i < kHeld / 2; ++i) t[i] = add2(t[i], q[i]);
        }
        if (on) Held<X, VEC>::template store<G>(dxs.row(a.rows, r), lane, packs, t);
    }
    if (!partial) return;
    cp_async_wait<0>();
    __syncthreads();  // the sums take the ring's place
    // column c of a row is element c % VEC of pack c / VEC
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int pack = lane + i / VEC * G;
        float e, f, g, h;
        unpack2(dw[i / 2], e, f);
        unpack2(db[i / 2], g, h);
        if (pack < packs) {
            float *to = sums + group * (2 * kHeld * G) + pack * VEC + i % VEC;
            to[0] = i & 1 ? f : e;
            to[kHeld * G] = i & 1 ? h : g;
        }
    }
    __syncthreads();
    const int dim = static_cast<int>(a.dim);
    for (int i = threadIdx.x; i < 2 * dim; i += kBackThreads) {
        const int which = i >= dim, c = i - which * dim;
        float v = 0.0f;
        for (int k = 0; k < kGroups; ++k) v = __fadd_rn(v, sums[(2 * k + which) * (kHeld * G) + c]);
        partial[static_cast<int64_t>(blockIdx.x) * 2 * dim + i] = v;
    }
}

}  // namespace ea

using namespace ea;

struct ea_layernorm {
    ea_layernorm_config cfg{};
    DeviceOf dev;
    cudaStream_t stream = nullptr;
    float *partial = nullptr;
};

namespace {

// Most parts that the rows of a call are summed in: enough for kPartCtas CTAs per SM together with the tiles of columns.
constexpr int kPartCtas = 8;
constexpr int64_t kMostHeld = kBackThreads * kHeld;                   // longer rows go the way of any width
constexpr int kSumsBytes = kBackThreads * kHeld * 2 * sizeof(float);
constexpr int kForwardThreads = 768;                                  // of an SM
int64_t max_parts(const ea_layernorm_config &c)
{
    if (c.dim <= kBackThreads * kHeld) return std::min<int64_t>(kMaxSms, std::max<int64_t>(c.max_rows, 1));  // one a CTA
    return std::clamp<int64_t>(kMaxSms * kPartCtas / over<int64_t>(c.dim, kColumnLanes), 1, over<int64_t>(std::max<int64_t>(c.max_rows, 1), kColumnRows));
}

int validate(const ea_layernorm_config *cfg)
{
    if (!cfg) return lm_fail(EA_E_INVAL, "config is NULL");
    if (cfg->dim < 1 || cfg->dim > (int64_t{1} << 20)) return lm_fail(EA_E_INVAL, "dim must be in [1, 2^20]");
    if (cfg->max_rows < 0 || cfg->max_rows > kMaxRows) return lm_fail(EA_E_INVAL, "max_rows must be in [0, 2^30]");
    if (!(cfg->eps >= 1e-30f) || !std::isfinite(cfg->eps)) return lm_fail(EA_E_INVAL, "eps must be finite and at least 1e-30");
    return EA_OK;
}

size_t layernorm_bytes(const ea_layernorm_config &c) { return up256(static_cast<size_t>(max_parts(c)) * 2 * c.dim * 4); }

// Checks what the two calls share; y: of the forward call, or dy.
int check_call(const ea_layernorm *h, const ea_layernorm_call *c, const void *x, const void *w, const void *b, const void *y, LnArgs &a)
{
    if (!h) return lm_fail(EA_E_INVAL, "handle is NULL");
    if (!c) return lm_fail(EA_E_INVAL, "call is NULL");
    if (c->outer < 0 || c->inner < 0 || (c->inner && c->outer > h->cfg.max_rows / c->inner))
        return lm_fail(EA_E_INVAL, "%lld x %lld rows: the handle takes up to %lld", static_cast<long long>(c->outer), static_cast<long long>(c->inner),
                       static_cast<long long>(h->cfg.max_rows));
    if (!is_float_type(c->x_type)) return lm_fail(EA_E_INVAL, "unknown type %d of x", c->x_type);
    if (!is_float_type(c->y_type)) return lm_fail(EA_E_INVAL, "unknown type %d of y", c->y_type);
    if (c->x_type != c->y_type && c->x_type != EA_T_F32) return lm_fail(EA_E_UNSUPPORTED, "x of 16 bits with y of another type");
    if ((w || b) && !is_float_type(c->weight_type)) return lm_fail(EA_E_INVAL, "unknown type %d of the weight", c->weight_type);
    int r = EA_OK;
    if (c->outer * c->inner) {
        r = check_address(x, c->x_type, "x");
        if (r == EA_OK) r = check_address(y, c->y_type, "y");
    }
    if (r == EA_OK && w) r = check_address(w, c->weight_type, "the weight");
    if (r == EA_OK && b) r = check_address(b, c->weight_type, "the bias");
    if (r == EA_OK) r = h->dev.check();
    if (r != EA_OK) return r;
    a = LnArgs{};
    a.n = static_cast<uint32_t>(c->outer * c->inner);
    a.dim = h->cfg.dim;
    a.eps = h->cfg.eps;
    a.inverse = static_cast<float>(1.0 / static_cast<double>(a.dim));
    a.w = w;
    a.b = b;
    a.weight_type = c->weight_type;
    a.grad_type = c->grad_type;
    if (c->inner > 1 && c->outer > 1) a.rows = rows_of(c->inner);
    return EA_OK;
}

// f(std::integral_constant<int, G>) for the smallest group that holds a row of dim elements.
template <class F>
void with_group(int64_t dim, F f)
{
    if (dim <= 4 * kHeld) f(std::integral_constant<int, 4>());
    else if (dim <= 8 * kHeld) f(std::integral_constant<int, 8>());
    else if (dim <= 16 * kHeld) f(std::integral_constant<int, 16>());
    else if (dim <= 32 * kHeld) f(std::integral_constant<int, 32>());
    else if (dim <= 64 * kHeld) f(std::integral_constant<int, 64>());
    else if (dim <= 128 * kHeld) f(std::integral_constant<int, 128>());
    else if (dim <= 256 * kHeld) f(std::integral_constant<int, 256>());
    else f(std::integral_constant<int, 512>());
}

// A tensor's rows; where the call has one row in a sequence or one sequence, the rows of the other direction.
template <class T>
RowsOf<T> rows_at(const ea_layernorm_call *c, const void *p, int64_t outer, int64_t inner)
{
    return RowsOf<T>{static_cast<T *>(const_cast<void *>(p)), outer, c->inner == 1 ? outer : inner};
}

}  // namespace

extern "C" {

int ea_layernorm_workspace_bytes(const ea_layernorm_config *cfg, size_t *bytes)
{
    if (!bytes) return lm_fail(EA_E_INVAL, "bytes is NULL");
    const int r = validate(cfg);
    if (r != EA_OK) return r;
    *bytes = layernorm_bytes(*cfg);
    return EA_OK;
}

int ea_layernorm_init(const ea_layernorm_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_layernorm **out)
{
    if (!out) return lm_fail(EA_E_INVAL, "out is NULL");
    *out = nullptr;
    int r = validate(cfg);
    if (r != EA_OK) return r;
    if ((r = check_workspace(workspace, workspace_bytes, layernorm_bytes(*cfg))) != EA_OK) return r;
    DeviceOf dev;
    if ((r = dev.query()) != EA_OK) return r;
    dev.sms = std::min(dev.sms, kMaxSms);
    ea_layernorm *h = new (std::nothrow) ea_layernorm;
    if (!h) return lm_fail(EA_E_INVAL, "out of host memory");
    h->cfg = *cfg;
    h->dev = dev;
    h->stream = static_cast<cudaStream_t>(stream);
    h->partial = static_cast<float *>(workspace);
    *out = h;
    return EA_OK;
}

int ea_layernorm_forward(ea_layernorm *h, const ea_layernorm_call *c, const void *x, const void *w, const void *b, void *y, float *stats)
{
    LnArgs a;
    int r = check_call(h, c, x, w, b, y, a);
    if (r == EA_OK) r = check_rows_apart(c->outer, c->inner, c->y_outer, c->y_inner, a.dim, "y");
    if (r == EA_OK && stats && reinterpret_cast<uintptr_t>(stats) % 8) r = lm_fail(EA_E_ALIGN, "stats is not aligned to its pairs");
    if (r != EA_OK || a.n == 0) return r;
    cudaError_t e = cudaSuccess;
    with_pair(c->x_type, c->y_type, [&](auto *xt, auto *yt) {
        using X = std::remove_reference_t<decltype(*xt)>;
        using Y = std::remove_reference_t<decltype(*yt)>;
        if constexpr (std::is_same<X, Y>::value || std::is_same<X, float>::value) {
            const RowsOf<const X> xs = rows_at<const X>(c, x, c->x_outer, c->x_inner);
            const RowsOf<Y> ys = rows_at<Y>(c, y, c->y_outer, c->y_inner);
            if (a.dim > kMostHeld) {
                ln_forward_any_kernel<X, Y><<<std::min<unsigned>(a.n, h->dev.sms * 8), kNormRowThreads, 0, h->stream>>>(a, xs, ys, stats);
                return;
            }
            constexpr int kVec = 16 / sizeof(X);
            const bool wide = rows_on(16, x, c->x_type, a.dim, c->outer, c->inner, c->x_outer, c->x_inner) &&
                              rows_on(kVec * sizeof(Y), y, c->y_type, a.dim, c->outer, c->inner, c->y_outer, c->y_inner);
            with_group(a.dim, [&](auto group) {
                constexpr int G = decltype(group)::value, kThreads = G > 32 ? G : 128;
                const uint32_t ctas = over<uint32_t>(a.n, kThreads / G), most = h->dev.sms * (kForwardThreads / kThreads);
                auto kernel = wide ? ln_forward_kernel<X, Y, kVec, G> : ln_forward_kernel<X, Y, 1, G>;
                const int ring = wide ? kForwardDepth * kThreads * kHeld * static_cast<int>(sizeof(X)) : 0;
                if (ring > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ring);
                if (e == cudaSuccess) kernel<<<std::min(ctas, most), kThreads, ring, h->stream>>>(a, xs, ys, stats);
            });
        }
    });
    return lm_cuda(e == cudaSuccess ? cudaGetLastError() : e, "launch");
}

int ea_layernorm_backward(ea_layernorm *h, const ea_layernorm_call *c, const void *dy, const void *x, const float *stats, const void *w,
                          const void *add, void *dx, void *dw, void *db, int32_t accumulate)
{
    if (accumulate != 0 && accumulate != 1) return lm_fail(EA_E_INVAL, "accumulate is 0 or 1");
    LnArgs a;
    int r = check_call(h, c, x, w, nullptr, dy, a);
    if (r != EA_OK) return r;
    if ((dw || db) && !is_float_type(c->grad_type)) return lm_fail(EA_E_INVAL, "unknown type %d of the weight's gradient", c->grad_type);
    if (dw) r = check_address(dw, c->grad_type, "dw");
    if (r == EA_OK && db) r = check_address(db, c->grad_type, "db");
    if (r == EA_OK && dw && dw == db) r = lm_fail(EA_E_INVAL, "dw and db are one");
    if (r == EA_OK && dx) r = check_address(dx, c->x_type, "dx");
    if (r == EA_OK && dx && add) r = check_address(add, c->x_type, "add");
    if (r == EA_OK && dx) r = check_rows_apart(c->outer, c->inner, c->dx_outer, c->dx_inner, a.dim, "dx");
    if (r == EA_OK && a.n && !stats) r = lm_fail(EA_E_INVAL, "stats is NULL");
    if (r == EA_OK && reinterpret_cast<uintptr_t>(stats) % 8) r = lm_fail(EA_E_ALIGN, "stats is not aligned to its pairs");
    if (r != EA_OK) return r;
    int parts = 0;
    cudaError_t e = cudaSuccess;
    with_pair(c->x_type, c->y_type, [&](auto *xt, auto *yt) {
        using X = std::remove_reference_t<decltype(*xt)>;
        using Y = std::remove_reference_t<decltype(*yt)>;
        if constexpr (std::is_same<X, Y>::value || std::is_same<X, float>::value) {
            if (!a.n) return;
            const RowsOf<const Y> dys = rows_at<const Y>(c, dy, c->y_outer, c->y_inner);
            const RowsOf<const X> xs = rows_at<const X>(c, x, c->x_outer, c->x_inner);
            const RowsOf<const X> adds = rows_at<const X>(c, add, c->add_outer, c->add_inner);
            const RowsOf<X> dxs = rows_at<X>(c, dx, c->dx_outer, c->dx_inner);
            if (a.dim > kMostHeld) {
                if (dw || db) {  // before dx, which may be in the place of dy or x
                    const int64_t most = max_parts(h->cfg), part = over<int64_t>(over<int64_t>(a.n, most), kColumnRows) * kColumnRows;
                    parts = static_cast<int>(over<int64_t>(a.n, part));
                    const dim3 grid(static_cast<unsigned>(over<int64_t>(a.dim, kColumnLanes)), parts);
                    ln_columns_any_kernel<X, Y><<<grid, dim3(kColumnLanes, kColumnRows), 0, h->stream>>>(a, dys, xs, stats, static_cast<uint32_t>(part), h->partial);
                }
                if (dx) ln_dx_any_kernel<X, Y><<<std::min<unsigned>(a.n, h->dev.sms * 8), kNormRowThreads, 0, h->stream>>>(a, dys, xs, stats, adds, dxs);
                return;
            }
            if (!dx && !dw && !db) return;
            constexpr int kVec = 16 / sizeof(X);
            auto on = [&](const void *p, int32_t type, int64_t outer, int64_t inner) {
                return rows_on(kVec * type_bytes(type), p, type, a.dim, c->outer, c->inner, outer, inner);
            };
            const bool wide = on(x, c->x_type, c->x_outer, c->x_inner) && on(dy, c->y_type, c->y_outer, c->y_inner) &&
                              (!dx || on(dx, c->x_type, c->dx_outer, c->dx_inner)) && (!dx || !add || on(add, c->x_type, c->add_outer, c->add_inner));
            with_group(a.dim, [&](auto group) {
                constexpr int G = decltype(group)::value;
                const uint32_t ctas = std::min<uint32_t>(over<uint32_t>(a.n, kBackThreads / G), h->dev.sms);
                float *partial = dw || db ? h->partial : nullptr;
                if (partial) parts = static_cast<int>(ctas);
                auto kernel = wide ? ln_backward_kernel<X, Y, kVec, G> : ln_backward_kernel<X, Y, 1, G>;
                const int ring = wide ? kBackDepth<X, Y> * kBackThreads * kHeld * (2 * static_cast<int>(sizeof(X)) + static_cast<int>(sizeof(Y))) : kSumsBytes;
                e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ring);
                if (e == cudaSuccess) kernel<<<ctas, kBackThreads, ring, h->stream>>>(a, dys, xs, stats, adds, dxs, partial);
            });
        }
    });
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess && (dw || db) && !(accumulate && !a.n)) {
        const dim3 grid(static_cast<unsigned>(over<int64_t>(a.dim, kColumnLanes)), 2);
        e = launch_lm(ln_join_kernel, grid, kColumnLanes * kColumnRows, 0, h->stream, a.n != 0, 1, a, static_cast<const float *>(h->partial), parts, dw, db,
                      static_cast<int>(accumulate));
    }
    return lm_cuda(e, "launch");
}

int ea_layernorm_destroy(ea_layernorm *h)
{
    delete h;
    return EA_OK;
}

}  // extern "C"
