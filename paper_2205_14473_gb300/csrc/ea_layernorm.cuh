// ea_layernorm.cuh -- what the layer norm and its gradient share: rows in registers, and the checks of a call.
//
// Both are one pass over the rows.  A group of lanes or warps holds a row in registers, 16 elements a thread, and the next rows are
// on their way to shared memory while it works on this one.  Rows that registers do not hold are read from the caches again.
#pragma once

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

// ---------------------------------------------------------------------------------------------- rows in registers
constexpr int kHeld = 16;                // elements of a thread
constexpr int kBackThreads = 512;
constexpr int kForwardDepth = 4;         // rows on their way
// Of the gradient: what 192 KB hold of x, dy and the added rows.
template <class X, class Y>
constexpr int kBackDepth = 192 * 1024 / (kBackThreads * kHeld * (2 * static_cast<int>(sizeof(X)) + static_cast<int>(sizeof(Y))));

// An asynchronous copy global -> shared of BYTES (8 or 16) bytes, of which the first `have` are read and the others 0.
template <int BYTES>
__device__ __forceinline__ void cp_async_first(void *dst, const void *src, int have)
{
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(have) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(have) : "memory");
}

// Where a row lies among the packs that its group reads: from element `off` of pack 0 to before element `end`.  Rows that are
// whole packs start at 0.  Rows that do not start on a pack's boundary (SHIFT) are read from the boundary before them, and a
// group's rows all lie `off` behind one: it takes every 8 m-th row.
template <int VEC, bool SHIFT>
struct Span {
    int off, end, packs;

    __device__ __forceinline__ Span(int dim, int shift) : off(SHIFT ? shift : 0), end(off + dim), packs(SHIFT ? (end + VEC - 1) / VEC : dim / VEC) {}
    // whether element j of pack i is one of the row's, for a pack below `packs`
    __device__ __forceinline__ bool has(int i, int j) const { return !SHIFT || static_cast<unsigned>(i * VEC + j - off) < static_cast<unsigned>(end - off); }
    __device__ __forceinline__ bool whole(int i) const { return !SHIFT || (i * VEC >= off && (i + 1) * VEC <= end); }
};

// A thread's 16 elements of a row: packs of VEC, pack k of lane l of a group of G being pack l + k G of the row.
template <class T, int VEC>
struct Held {
    struct alignas(VEC * sizeof(T)) Pack {
        T x[VEC];
    };
    static constexpr int kPacks = kHeld / VEC;
    Pack p[kPacks];

    // A row's packs on their way to `slots`, every kStep-th of which is the thread's, zeros behind the row.  What lies in pack 0
    // before the row is the end of the row before it; the first row of a tensor has none.
    template <int G, int kStep, class S>
    static __device__ __forceinline__ void fetch(Pack *slots, const T *row, int lane, const S &span, const T *tensor)
    {
        const T *from = row - span.off;
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const int i = lane + k * G;
            if (i >= span.packs) continue;
            if (span.whole(i)) {
                if constexpr (sizeof(Pack) == 16) cp_async16(slots + k * kStep, from + i * VEC);
                else cp_async_first<sizeof(Pack)>(slots + k * kStep, from + i * VEC, sizeof(Pack));
            } else if (from + i * VEC >= tensor) {
                cp_async_first<sizeof(Pack)>(slots + k * kStep, from + i * VEC, min(span.end - i * VEC, VEC) * static_cast<int>(sizeof(T)));
            } else {
#pragma unroll 1
                for (int j = 0; j < VEC; ++j) slots[k * kStep].x[j] = span.has(i, j) ? from[i * VEC + j] : from_f32<T>(0.0f);
            }
        }
    }
    template <int kStep>
    static __device__ __forceinline__ void clear(Pack *slots)
    {
#pragma unroll
        for (int k = 0; k < kPacks; ++k) slots[k * kStep] = Pack{};
    }
    template <int kStep, class S>
    __device__ __forceinline__ void take(const Pack *slots, int lane, const S &span)
    {
#pragma unroll
        for (int k = 0; k < kPacks; ++k) p[k] = slots[k * kStep];
        if (lane == 0 && span.off)
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (j < span.off) p[0].x[j] = from_f32<T>(0.0f);
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
    template <int G, class S>
    static __device__ __forceinline__ void store(T *row, int lane, const S &span, const F2 (&y)[kHeld / 2])
    {
        T *to = row - span.off;
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
            const int i = lane + k * G;
            if (i >= span.packs) continue;
            if (span.whole(i)) {
                reinterpret_cast<Pack *>(to)[i] = q;
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (span.has(i, j)) to[i * VEC + j] = q.x[j];
            }
        }
    }
};

// The same elements of a weight of any type and alignment; `fill` for a weight that is NULL and outside the row.
template <int G, int VEC, bool SHIFT>
__device__ __forceinline__ void load_weight(const void *w, int32_t type, int lane, const Span<VEC, SHIFT> &span, float fill, F2 (&y)[kHeld / 2])
{
    float f[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int pack = lane + i / VEC * G;
        f[i] = w && pack < span.packs && span.has(pack, i % VEC) ? load_any(w, type, pack * VEC + i % VEC - span.off) : fill;
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
// 1 / sqrt of a number of at least 1e-30: the hardware's approximation and one Newton step.
__device__ __forceinline__ float rsqrt_of(float x)
{
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    const float h = __fmul_rn(__fmul_rn(-0.5f, x), y);
    return x < __int_as_float(0x7f800000) ? __fmaf_rn(__fmaf_rn(h, y, 0.5f), y, y) : y;
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

// How far behind a pack's boundary a row starts.
template <int VEC, class T>
__device__ __forceinline__ int phase_of(const RowsOf<T> &t, const Rows &rows, uint32_t r)
{
    return static_cast<int>(reinterpret_cast<uintptr_t>(t.row(rows, r)) / sizeof(T) % VEC);
}

}  // namespace ea

struct ea_layernorm {
    ea_layernorm_config cfg{};
    ea::DeviceOf dev;
    cudaStream_t stream = nullptr;
    float *partial = nullptr;
    ea::Allowed allowed;
};

namespace ea {

// Most parts that the rows of a call are summed in: enough for kPartCtas CTAs per SM together with the tiles of columns.
constexpr int kPartCtas = 8;
constexpr int64_t kMostHeld = kBackThreads * kHeld;                   // longer rows go the way of any width
constexpr int kSumsBytes = kBackThreads * kHeld * 2 * sizeof(float);
constexpr int kForwardThreads = 768;                                  // of an SM
inline int64_t max_parts(const ea_layernorm_config &c)
{
    if (c.dim <= kBackThreads * kHeld) return std::min<int64_t>(kMaxSms, std::max<int64_t>(c.max_rows, 1));  // one a CTA
    return std::clamp<int64_t>(kMaxSms * kPartCtas / over<int64_t>(c.dim, kColumnLanes), 1, over<int64_t>(std::max<int64_t>(c.max_rows, 1), kColumnRows));
}

inline int validate(const ea_layernorm_config *cfg)
{
    if (!cfg) return lm_fail(EA_E_INVAL, "config is NULL");
    if (cfg->dim < 1 || cfg->dim > (int64_t{1} << 20)) return lm_fail(EA_E_INVAL, "dim must be in [1, 2^20]");
    if (cfg->max_rows < 0 || cfg->max_rows > kMaxRows) return lm_fail(EA_E_INVAL, "max_rows must be in [0, 2^30]");
    if (!(cfg->eps >= 1e-30f) || !std::isfinite(cfg->eps)) return lm_fail(EA_E_INVAL, "eps must be finite and at least 1e-30");
    return EA_OK;
}

inline size_t layernorm_bytes(const ea_layernorm_config &c) { return up256(static_cast<size_t>(max_parts(c)) * 2 * c.dim * 4); }

// Checks what the two calls share; y: of the forward call, or dy.
inline int check_call(const ea_layernorm *h, const ea_layernorm_call *c, const void *x, const void *w, const void *b, const void *y, LnArgs &a)
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

template <int N>
using Int = std::integral_constant<int, N>;

// f(Int<G>) for the smallest group that holds a row of dim elements.
template <class F>
void with_group(int64_t dim, F f)
{
    if (dim <= 4 * kHeld) f(Int<4>());
    else if (dim <= 8 * kHeld) f(Int<8>());
    else if (dim <= 16 * kHeld) f(Int<16>());
    else if (dim <= 32 * kHeld) f(Int<32>());
    else if (dim <= 64 * kHeld) f(Int<64>());
    else if (dim <= 128 * kHeld) f(Int<128>());
    else if (dim <= 256 * kHeld) f(Int<256>());
    else f(Int<512>());
}

// How a call's rows can be read: in whole packs of VEC elements, in packs from the boundary before them, or one by one.
enum Access { kWhole, kShifted, kSingle };

struct AccessOf {
    const ea_layernorm_call *c;
    int64_t dim, vec;
    bool whole = true, flat = true, alike = true;
    int64_t phase = -1, step = 0;

    void add(const void *p, int32_t type, int64_t outer, int64_t inner)
    {
        whole = whole && rows_on(vec * type_bytes(type), p, type, dim, c->outer, c->inner, outer, inner);
        flat = flat && (c->outer <= 1 || c->inner <= 1 || outer == c->inner * inner);
        const int64_t at = static_cast<int64_t>(reinterpret_cast<uintptr_t>(p) / type_bytes(type) % vec), by = (c->inner > 1 ? inner : outer) % vec;
        alike = alike && (phase < 0 || (at == phase && by == step));
        phase = at, step = by;
    }
    // binary32 elements are read one by one as fast (7,021 x 769, gradient: 19.6 us; shifted 23.3)
    Access get() const { return whole ? kWhole : vec > 4 && flat && alike && dim + vec - 1 <= kMostHeld ? kShifted : kSingle; }
};

// f(Int<G>, Int<VEC>, whether shifted) for an access of packs of VEC.
template <int VEC, class F>
void with_rows(int64_t dim, Access access, F f)
{
    if (access == kWhole) with_group(dim, [&](auto group) { f(group, Int<VEC>(), std::false_type()); });
    else if (access == kShifted) {
        if constexpr (VEC > 4) with_group(dim + VEC - 1, [&](auto group) { f(group, Int<VEC>(), std::true_type()); });
    } else with_group(dim, [&](auto group) { f(group, Int<1>(), std::false_type()); });
}

// A tensor's rows; where the call has one row in a sequence or one sequence, the rows of the other direction.
template <class T>
RowsOf<T> rows_at(const ea_layernorm_call *c, const void *p, int64_t outer, int64_t inner)
{
    return RowsOf<T>{static_cast<T *>(const_cast<void *>(p)), outer, c->inner == 1 ? outer : inner};
}

}  // namespace ea
