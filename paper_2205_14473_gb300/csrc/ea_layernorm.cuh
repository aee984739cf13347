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
constexpr int kForwardDepth = 3;         // rows on their way
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

    // A row's packs on their way to `slots`, every kStep-th of which is the thread's.
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
        f[i] = w && pack < packs ? load_any(w, type, pack * VEC + i % VEC) : fill;
    }
#pragma unroll
    for (int i = 0; i < kHeld / 2; ++i) y[i] = pack2(f[2 * i], f[2 * i + 1]);
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

// Whether a call's rows are whole packs of VEC elements, each on its boundary, and whether they follow one another at one
// distance, whatever sequence they are in.
struct RowsLie {
    const ea_layernorm_call *c;
    int64_t dim, vec;
    bool whole = true, flat = true;

    void add(const void *p, int32_t type, int64_t outer, int64_t inner)
    {
        whole = whole && rows_on(vec * type_bytes(type), p, type, dim, c->outer, c->inner, outer, inner);
        flat = flat && (c->outer <= 1 || c->inner <= 1 || outer == c->inner * inner);
    }
};

// f(Int<G>, Int<elements of a pack>) for rows in packs of VEC, or one element after the other.
template <int VEC, class F>
void with_rows(int64_t dim, bool whole, F f)
{
    with_group(dim, [&](auto group) {
        if (whole) f(group, Int<VEC>());
        else f(group, Int<1>());
    });
}

// A tensor's rows; where the call has one row in a sequence or one sequence, the rows of the other direction.
template <class T>
RowsOf<T> rows_at(const ea_layernorm_call *c, const void *p, int64_t outer, int64_t inner)
{
    return RowsOf<T>{static_cast<T *>(const_cast<void *>(p)), outer, c->inner == 1 ? outer : inner};
}

}  // namespace ea
