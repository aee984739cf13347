// ea_adamw.cu -- ea_adamw_step: one AdamW step (Loshchilov and Hutter; Adam's bias correction folded into the
// step size and epsilon as in the last remark of Kingma and Ba's Section 2) over a list of tensors, with
// moments in binary32 or in 8 bits.
#include <cuda_fp8.h>

#include <type_traits>

#include "ea_lm.cuh"

namespace ea {

constexpr int kAdamThreads = 256;
constexpr int kAdamCtasPerSm = 2;  // 128 registers per thread; a persistent grid of them
constexpr int kBlock = EA_ADAMW_BLOCK;  // a warp's unit of work: eight coordinates per lane

// What a step needs to know of the steps before it.  The last CTA of a step that is not skipped advances it.
struct AdamState {
    int64_t t;        // steps taken
    double b1, b2;    // beta1^(t+1), beta2^(t+1)
    float a, e;       // sqrt(1 - b2) / (1 - b1) and eps sqrt(1 - b2): the coming step's, rounded once
    unsigned ticket;  // CTAs of the current step that are done
    unsigned pad;
};

struct AdamArgs {
    int64_t units;                 // blocks of this launch's tensors
    int n_tensors, tensor0;        // this launch's tensors, and the first one's index
    const int64_t *first;          // n_tensors + 1: each tensor's first block within the launch
    const ea_adamw_tensor *tensors;
    AdamState *state;
    int last;                      // whether this launch is the step's last
    float lr, beta1, beta2, c1, c2;
    double beta1d, beta2d, eps;
    const float *clip;
    uint2 keys[10];                // Philox's key of every round
    float minus_zero;              // -0 (see mul2)
};

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
__device__ __forceinline__ F2 both(float a) { return pack2(a, a); }
// a b as a b + (-0), the same value, with a -0 that the compiler does not know: a packed product and the packed sum
// after it would be merged into one rounding, whatever their PTX says.
__device__ __forceinline__ F2 mul2(F2 a, F2 b, F2 minus_zero) { return fma2(a, b, minus_zero); }

__device__ __forceinline__ F2 negate2(F2 a) { return F2{a.v ^ 0x8000000080000000ull}; }

// Within 2^-23 relative of the reciprocal of a normal number.
__device__ __forceinline__ float recip_normal(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// The square roots of two numbers, zero or normal, rounded to nearest: from y ~ 1 / sqrt(x), g = x y and h = y / 2
// are refined together (Goldschmidt), g <- g + g (1/2 - g h), h <- h + h (1/2 - g h), and the remainder x - g^2,
// exact in a fused operation, corrects g's last bit (Markstein, "Computation of elementary functions on the IBM
// RISC System/6000 processor", 1990).  Equal to sqrtf for every number above 2^-100.  It is half the
// instructions of two calls, and no branch stands between the eight coordinates of a lane.
__device__ __forceinline__ void sqrt_pair(float &a, float &b)
{
    float ya, yb;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(ya) : "f"(fmaxf(a, 0x1p-126f)));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(yb) : "f"(fmaxf(b, 0x1p-126f)));
    const F2 x = pack2(a, b), y = pack2(ya, yb);
    const F2 none = both(-0.0f);  // nothing here may be merged to another effect: every sum is a fused one already
    F2 g = fma2(x, y, none), h = fma2(y, both(0.5f), none);
    const F2 e = fma2(negate2(g), h, both(0.5f));
    g = fma2(g, e, g);
    h = fma2(h, e, h);
    g = fma2(fma2(negate2(g), g, x), h, g);
    unpack2(g, a, b);
}

// Philox4x32-10 with the round keys formed once on the host.
__device__ __forceinline__ uint4 philox_words(uint4 c, const uint2 (&keys)[10])
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = static_cast<uint64_t>(0xD2511F53u) * c.x, p1 = static_cast<uint64_t>(0xCD9E8D57u) * c.z;
        c = make_uint4(static_cast<uint32_t>(p1 >> 32) ^ c.y ^ keys[r].x, static_cast<uint32_t>(p1),
                       static_cast<uint32_t>(p0 >> 32) ^ c.w ^ keys[r].y, static_cast<uint32_t>(p0));
    }
    return c;
}

// The values of four e4m3 codes, exact.
__device__ __forceinline__ void e4m3_values(uint32_t codes, float (&x)[4])
{
    const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes & 0xffffu), __NV_E4M3);
    const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes >> 16), __NV_E4M3);
    const float2 lo = __half22float2(__half2(a)), hi = __half22float2(__half2(b));
    x[0] = lo.x, x[1] = lo.y, x[2] = hi.x, x[3] = hi.y;
}

// Four consecutive elements as they lie in memory: one 16-, 8- or 4-byte access.
template <class T>
struct alignas(4 * sizeof(T)) Quad {
    T x[4];
};

// Those from p on, where `whole`, else the ones below n (the others are 0).
template <class T>
__device__ __forceinline__ Quad<T> load_quad(const T *p, int n, bool whole)
{
    using Word = typename std::conditional<sizeof(T) == 4, uint4, typename std::conditional<sizeof(T) == 2, uint2, uint32_t>::type>::type;
    union {
        Word w;
        Quad<T> q;
    } v{};
    if (whole) {
        v.w = *reinterpret_cast<const Word *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) v.q.x[i] = p[i];
    }
    return v.q;
}
template <class T>
__device__ __forceinline__ void store_quad(T *p, int n, bool whole, const Quad<T> &q)
{
    using Word = typename std::conditional<sizeof(T) == 4, uint4, typename std::conditional<sizeof(T) == 2, uint2, uint32_t>::type>::type;
    if (whole) {
        *reinterpret_cast<Word *>(p) = *reinterpret_cast<const Word *>(&q);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = q.x[i];
    }
}
template <class T>
__device__ __forceinline__ void quad_values(const Quad<T> &q, float (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = to_f32(q.x[i]);
}
template <class T>
__device__ __forceinline__ Quad<T> quad_of(const float (&x)[4])
{
    Quad<T> q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.x[i] = from_f32<T>(x[i]);
    return q;
}

// The exponent k of the smallest power of two >= 2^-126 with amax / 2^k <= 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(uint32_t amax_bits)
{
    return max(static_cast<int>((amax_bits + 0x1fffffu) >> 23) - 127 - 8, -126);
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float(static_cast<uint32_t>(127 + k) << 23); }

// |x|'s bits, which order as it does; 0 where it is not finite.
__device__ __forceinline__ uint32_t finite_magnitude(float x)
{
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// A step's arithmetic on four coordinates, in packed pairs.
struct AdamStep {
    float factor, beta1, beta2, c1, c2, e, step, rate;
    F2 z;  // (-0, -0)

    // The new parameters, from the moments and the second one's root (times `unit`, a power of two).
    __device__ __forceinline__ void params(float (&p)[4], const float (&m)[4], const float (&root)[4], float unit) const
    {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            float d0, d1;
            unpack2(fma2(pack2(root[i], root[i + 1]), both(unit), both(e)), d0, d1);
            const F2 q = mul2(pack2(m[i], m[i + 1]), pack2(recip_normal(d0), recip_normal(d1)), z);
            const F2 x = pack2(p[i], p[i + 1]), d = add2(mul2(x, both(rate), z), mul2(q, both(step), z));
            unpack2(fma2(d, both(-1.0f), x), p[i], p[i + 1]);
        }
    }

    // m <- mb m + c1 g and v <- vb v + c2 g^2 with g the gradient times the factor.
    __device__ __forceinline__ void moments(float (&m)[4], float (&v)[4], const float (&grad)[4], float mb, float vb) const
    {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const F2 g = mul2(pack2(grad[i], grad[i + 1]), both(factor), z);
            unpack2(add2(mul2(pack2(m[i], m[i + 1]), both(mb), z), mul2(g, both(c1), z)), m[i], m[i + 1]);
            unpack2(add2(mul2(pack2(v[i], v[i + 1]), both(vb), z), mul2(mul2(g, g, z), both(c2), z)), v[i], v[i + 1]);
        }
    }
};

// Four magnitudes y <= 448 (but for the root's last bit, which saturates) in e4m3, rounded up with the probability
// of the remainder.  A normal number's 20 bits below its third mantissa bit get a random number added and are cut
// off; below 2^-6 the grid's spacing is 2^-9 throughout.  r: 16 random bits each, in bits 4 .. 19.
template <bool KEEP_NONZERO>
__device__ __forceinline__ void round_e4m3(float (&y)[4], const uint32_t (&r)[4])
{
    constexpr uint32_t kNormal = (127u - 6u) << 23;
    uint32_t least = 0xffffffffu;
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        q[i] = __uint_as_float((__float_as_uint(y[i]) + r[i]) & 0xfff00000u);
        least = min(least, __float_as_uint(y[i]) - 1u);
    }
    if (least < kNormal - 1u) {  // some 0 < y < 2^-6
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (__float_as_uint(y[i]) - 1u < kNormal - 1u) {
                const float up = __fmaf_rn(static_cast<float>(r[i]), 0x1p-20f, __fmul_rn(y[i], 512.0f));
                const float n = __fsub_rn(__fadd_rd(up, 0x1p23f), 0x1p23f);  // its floor
                q[i] = __fmul_rn(KEEP_NONZERO ? fmaxf(n, 1.0f) : n, 0x1p-9f);
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = q[i];
}

// Codes of four values of the format (the last one's in the highest byte); NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3_codes(const float (&x)[4])
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[1]), "f"(x[0]));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[3]), "f"(x[2]));
    return lo | static_cast<uint32_t>(hi) << 16;
}

// Where a warp stands: its block's tensor and addresses, and how much of the block there is.
template <class P, class G>
struct AdamCursor {
    int64_t u;       // block of the launch
    int64_t block;   // of the tensor
    int t, n;        // tensor; coordinates of the block
    bool vec;        // a whole block, every address aligned to four elements
    P *p;
    const G *g;
    void *m, *v;
};

// A block's loads: 4 coordinates in each half of the block per lane.
template <class P, class G, class S>
struct AdamBlock {
    Quad<P> p[2];
    Quad<G> g[2];
    Quad<S> m[2], v[2];
    float ms, vs;
};

// 8-bit states are handled as bytes, 32-bit ones as numbers.
template <int BITS>
using AdamCell = typename std::conditional<BITS == 32, float, uint8_t>::type;

template <int BITS, class P, class G, class C>
__device__ __forceinline__ void adam_seek(const AdamArgs &a, const GradList &list, int64_t u, AdamCursor<P, G> &c)
{
    using S = AdamCell<BITS>;
    c.t = tensor_of(a.first, a.n_tensors, u, c.t);
    const ea_adamw_tensor &T = a.tensors[c.t];
    c.u = u;
    c.block = u - a.first[c.t];
    const int64_t at = c.block * kBlock;
    c.n = static_cast<int>(min(T.size - at, static_cast<int64_t>(kBlock)));
    c.p = static_cast<P *>(T.param) + at;
    c.g = static_cast<const G *>(list.g[c.t]) + at;
    c.m = static_cast<S *>(T.m) + at;
    c.v = static_cast<S *>(T.v) + at;
    // (a block's offset keeps the alignment of its tensor)
    c.vec = c.n == kBlock && reinterpret_cast<uintptr_t>(c.p) % sizeof(Quad<P>) == 0 && reinterpret_cast<uintptr_t>(c.g) % sizeof(Quad<G>) == 0 &&
            reinterpret_cast<uintptr_t>(T.copy) % sizeof(Quad<C>) == 0 &&
            (reinterpret_cast<uintptr_t>(c.m) | reinterpret_cast<uintptr_t>(c.v)) % sizeof(Quad<S>) == 0;
}

template <int BITS, class P, class G>
__device__ __forceinline__ void adam_load(const AdamArgs &a, const AdamCursor<P, G> &c, AdamBlock<P, G, AdamCell<BITS>> &b)
{
    using S = AdamCell<BITS>;
    const int j0 = (threadIdx.x & 31) * 4;
    const S *m = static_cast<const S *>(c.m), *v = static_cast<const S *>(c.v);
    if (c.vec) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = j0 + 128 * h;
            b.p[h] = load_quad(c.p + j, 4, true);
            b.g[h] = load_quad(c.g + j, 4, true);
            b.m[h] = load_quad(m + j, 4, true);
            b.v[h] = load_quad(v + j, 4, true);
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = j0 + 128 * h;
            b.p[h] = load_quad(c.p + j, c.n - j, false);
            b.g[h] = load_quad(c.g + j, c.n - j, false);
            b.m[h] = load_quad(m + j, c.n - j, false);
            b.v[h] = load_quad(v + j, c.n - j, false);
        }
    }
    if constexpr (BITS == 8) {
        b.ms = a.tensors[c.t].m_scale[c.block];
        b.vs = a.tensors[c.t].v_scale[c.block];
    }
}

template <int BITS, class P, class G, class C>
__device__ __forceinline__ void adam_store(const AdamArgs &a, const AdamCursor<P, G> &c, const float (&p)[2][4],
                                           const Quad<AdamCell<BITS>> (&m)[2], const Quad<AdamCell<BITS>> (&v)[2])
{
    using S = AdamCell<BITS>;
    const int j0 = (threadIdx.x & 31) * 4;
    C *copy = static_cast<C *>(a.tensors[c.t].copy);
    if (copy) copy += c.block * kBlock;
    if (c.vec) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = j0 + 128 * h;
            store_quad(c.p + j, 4, true, quad_of<P>(p[h]));
            if (copy) store_quad(copy + j, 4, true, quad_of<C>(p[h]));
            store_quad(static_cast<S *>(c.m) + j, 4, true, m[h]);
            store_quad(static_cast<S *>(c.v) + j, 4, true, v[h]);
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = j0 + 128 * h, n = c.n - j;
            store_quad(c.p + j, n, false, quad_of<P>(p[h]));
            if (copy) store_quad(copy + j, n, false, quad_of<C>(p[h]));
            store_quad(static_cast<S *>(c.m) + j, n, false, m[h]);
            store_quad(static_cast<S *>(c.v) + j, n, false, v[h]);
        }
    }
}

// The 32-bit step of a block.
template <class P, class G, class C>
__device__ __forceinline__ void adam_block(const AdamArgs &a, const AdamState &, const AdamStep &s, const AdamCursor<P, G> &c,
                                           const AdamBlock<P, G, float> &b)
{
    float p[2][4];
    Quad<float> mq[2], vq[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float m[4], v[4], g[4], root[4];
        quad_values(b.p[h], p[h]);
        quad_values(b.g[h], g);
        quad_values(b.m[h], m);
        quad_values(b.v[h], v);
        s.moments(m, v, g, s.beta1, s.beta2);
#pragma unroll
        for (int i = 0; i < 4; ++i) root[i] = __fsqrt_rn(v[i]);
        s.params(p[h], m, root, 1.0f);
        mq[h] = quad_of<float>(m);
        vq[h] = quad_of<float>(v);
    }
    adam_store<32, P, G, C>(a, c, p, mq, vq);
}

// The 8-bit step of a block.
template <class P, class G, class C>
__device__ __forceinline__ void adam_block(const AdamArgs &a, const AdamState &st, const AdamStep &s, const AdamCursor<P, G> &c,
                                           const AdamBlock<P, G, uint8_t> &b)
{
    float m[2][4], v[2][4], p[2][4];
    Quad<uint8_t> mq[2], vq[2];
    // beta1 m scale and beta2 (r scale)^2 are one multiplication each where the power of two leaves the product
    // normal: a scale below 2^-40 goes into the values first
    const bool small = b.ms < 0x1p-40f || b.vs < 0x1p-40f;
    const float mb = small ? s.beta1 : __fmul_rn(s.beta1, b.ms), vb = small ? s.beta2 : __fmul_rn(s.beta2, __fmul_rn(b.vs, b.vs));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        e4m3_values(*reinterpret_cast<const uint32_t *>(&b.m[h]), m[h]);
        e4m3_values(*reinterpret_cast<const uint32_t *>(&b.v[h]), v[h]);
    }
    if (small)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i >> 2][i & 3] = __fmul_rn(m[i >> 2][i & 3], b.ms);
            v[i >> 2][i & 3] = __fmul_rn(v[i >> 2][i & 3], b.vs);
        }
    uint32_t am = 0, av = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float g[4];
        quad_values(b.g[h], g);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[h][i] = __fmul_rn(v[h][i], v[h][i]);
        s.moments(m[h], v[h], g, mb, vb);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            am = max(am, __float_as_uint(fabsf(m[h][i])));
            av = max(av, __float_as_uint(v[h][i]));
        }
    }
    am = __reduce_max_sync(0xffffffffu, am);
    av = __reduce_max_sync(0xffffffffu, av);
    const bool finite = max(am, av) < 0x7f800000u;
    if (!finite) {  // the scales go by the finite values; the others are held as NaN
        am = av = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            am = max(am, finite_magnitude(m[i >> 2][i & 3]));
            av = max(av, finite_magnitude(v[i >> 2][i & 3]));
        }
        am = __reduce_max_sync(0xffffffffu, am);
        av = __reduce_max_sync(0xffffffffu, av);
    }
    // roots are taken 2^32 times as large, so that subnormal values have one, where none overflows
    const bool lift = finite && av < (127u + 60u) << 23;
    const float unit = lift ? 0x1p-32f : 1.0f;
    const int km = scale_exponent(am), kv = scale_exponent(__float_as_uint(__fsqrt_rn(__uint_as_float(av))));
    const float im = power_of_two(-km), iv = __fmul_rn(power_of_two(-kv), unit);
    if ((threadIdx.x & 31) == 0) {
        a.tensors[c.t].m_scale[c.block] = power_of_two(km);
        a.tensors[c.t].v_scale[c.block] = power_of_two(kv);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float root[4];
        if (lift) {
#pragma unroll
            for (int i = 0; i < 4; ++i) root[i] = __fmul_rn(v[h][i], 0x1p64f);
            sqrt_pair(root[0], root[1]);
            sqrt_pair(root[2], root[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) root[i] = __fsqrt_rn(v[h][i]);
        }
        quad_values(b.p[h], p[h]);
        s.params(p[h], m[h], root, unit);
        const uint64_t quad = (static_cast<uint64_t>(c.block) * kBlock + 128 * h + (threadIdx.x & 31) * 4) >> 2;
        const uint4 w = philox_words(make_uint4(static_cast<uint32_t>(quad), static_cast<uint32_t>(quad >> 32),
                                                static_cast<uint32_t>(a.tensor0 + c.t), static_cast<uint32_t>(st.t)), a.keys);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
        float ym[4], yv[4];
        uint32_t rm[4], rv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ym[i] = __fmul_rn(fabsf(m[h][i]), im);
            yv[i] = __fmul_rn(root[i], iv);
            rm[i] = (word[i] << 4) & 0xffff0u;
            rv[i] = (word[i] >> 12) & 0xffff0u;
        }
        round_e4m3<false>(ym, rm);
        round_e4m3<true>(yv, rv);
#pragma unroll
        for (int i = 0; i < 4; ++i) ym[i] = copysignf(ym[i], m[h][i]);
        if (!finite)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!isfinite(m[h][i])) ym[i] = __int_as_float(0x7fc00000);
                if (!isfinite(v[h][i])) yv[i] = __int_as_float(0x7fc00000);
            }
        *reinterpret_cast<uint32_t *>(&mq[h]) = e4m3_codes(ym);
        *reinterpret_cast<uint32_t *>(&vq[h]) = e4m3_codes(yv);
    }
    adam_store<8, P, G, C>(a, c, p, mq, vq);
}

// A CTA takes a contiguous piece of the launch's blocks of 256 coordinates, its warps in turn: so a warp's tensor
// seldom changes, and every CTA has the same number of blocks but for one.  A lane holds four consecutive
// coordinates in each half of a block: every access of the warp is one contiguous piece, and the block's scale is
// one warp reduction.  The next block's loads are issued before this one's arithmetic, 8-bit states' 70
// instructions per coordinate.
template <class P, class G, class C, int BITS>
__global__ void __launch_bounds__(kAdamThreads, kAdamCtasPerSm) adamw_kernel(const __grid_constant__ AdamArgs a, const __grid_constant__ GradList list)
{
    constexpr int kWarps = kAdamThreads / 32;
    const float factor = a.clip ? a.clip[1] : 1.0f;
    const AdamState st = *a.state;
    const int64_t begin = a.units * blockIdx.x / gridDim.x, end = a.units * (blockIdx.x + 1) / gridDim.x;
    AdamCursor<P, G> c;
    c.t = 0;
    int64_t u = begin + (threadIdx.x >> 5);
    if (!isnan(factor) && u < end) {
        AdamStep s{factor, a.beta1, a.beta2, a.c1, a.c2, st.e, 0.0f, 0.0f, both(a.minus_zero)};
        AdamBlock<P, G, AdamCell<BITS>> b;
        adam_seek<BITS, P, G, C>(a, list, u, c);
        adam_load<BITS>(a, c, b);
        while (true) {
            const AdamCursor<P, G> now = c;
            const AdamBlock<P, G, AdamCell<BITS>> block = b;
            u += kWarps;
            if (u < end) {
                adam_seek<BITS, P, G, C>(a, list, u, c);
                adam_load<BITS>(a, c, b);
            }
            const float lr = __fmul_rn(a.lr, a.tensors[now.t].lr_scale);
            s.step = __fmul_rn(lr, st.a);
            s.rate = __fmul_rn(lr, a.tensors[now.t].weight_decay);
            adam_block<P, G, C>(a, st, s, now, block);
            if (u >= end) break;
        }
    }
    if (!a.last) return;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&a.state->ticket, 1u) == gridDim.x - 1) {
            a.state->ticket = 0;
            if (!isnan(factor)) {
                const double b1 = st.b1 * a.beta1d, b2 = st.b2 * a.beta2d, root = sqrt(1.0 - b2);
                a.state->t = st.t + 1;
                a.state->b1 = b1;
                a.state->b2 = b2;
                a.state->a = static_cast<float>(root / (1.0 - b1));
                a.state->e = static_cast<float>(a.eps * root);
            }
        }
    }
}

}  // namespace ea

using namespace ea;

struct ea_adamw {
    DeviceOf dev;
    cudaStream_t stream = nullptr;
    ea_adamw_config cfg{};
    std::vector<ea_adamw_tensor> tensors;
    struct Launch {
        int first_tensor, n_tensors, grid;
        int64_t units, first_at;
    };
    std::vector<Launch> launches;
    std::vector<int64_t> table;
    AdamState start{};
    int64_t *d_first = nullptr;
    ea_adamw_tensor *d_tensors = nullptr;
    AdamState *d_state = nullptr;
};

namespace {

int validate(const ea_adamw_config *cfg)
{
    if (!cfg) return lm_fail(EA_E_INVAL, "config is NULL");
    if (cfg->n_tensors < 1 || cfg->n_tensors > (1 << 20)) return lm_fail(EA_E_INVAL, "n_tensors must be in [1, 2^20]");
    if (!cfg->tensors) return lm_fail(EA_E_INVAL, "tensors is NULL");
    if (!is_float_type(cfg->param_type)) return lm_fail(EA_E_INVAL, "unknown parameter type %d", cfg->param_type);
    if (cfg->param_type == EA_T_F16) return lm_fail(EA_E_UNSUPPORTED, "parameters are binary32 or bfloat16");
    if (!is_float_type(cfg->grad_type)) return lm_fail(EA_E_INVAL, "unknown gradient type %d", cfg->grad_type);
    if (cfg->state_bits != 32 && cfg->state_bits != 8) return lm_fail(EA_E_INVAL, "state_bits is 32 or 8");
    if (!(cfg->beta1 >= 0.0f && cfg->beta1 < 1.0f)) return lm_fail(EA_E_INVAL, "beta1 must be in [0, 1)");
    if (!(cfg->beta2 >= 0.0f && cfg->beta2 < 1.0f)) return lm_fail(EA_E_INVAL, "beta2 must be in [0, 1)");
    if (!(cfg->eps >= 1e-30f) || !std::isfinite(cfg->eps)) return lm_fail(EA_E_INVAL, "eps must be >= 1e-30");
    if (cfg->step < 0 || cfg->step >= (int64_t{1} << 32)) return lm_fail(EA_E_INVAL, "step out of [0, 2^32)");
    const int32_t state = cfg->state_bits == 32 ? EA_T_F32 : -1;
    for (int32_t i = 0; i < cfg->n_tensors; ++i) {
        const ea_adamw_tensor &T = cfg->tensors[i];
        if (T.size < 0 || T.size > (int64_t{1} << 40)) return lm_fail(EA_E_INVAL, "the size of tensor %d is out of [0, 2^40]", i);
        if (!(T.weight_decay >= 0.0f) || !std::isfinite(T.weight_decay))
            return lm_fail(EA_E_INVAL, "the weight decay of tensor %d must be >= 0", i);
        if (!(T.lr_scale >= 0.0f) || !std::isfinite(T.lr_scale)) return lm_fail(EA_E_INVAL, "the lr_scale of tensor %d must be >= 0", i);
        if (T.size == 0) continue;
        int r = check_address(T.param, cfg->param_type, "a parameter");
        if (state == EA_T_F32) {
            if (r == EA_OK) r = check_address(T.m, EA_T_F32, "m");
            if (r == EA_OK) r = check_address(T.v, EA_T_F32, "v");
        } else {
            if (!T.m || !T.v) return lm_fail(EA_E_INVAL, "m or v of tensor %d is NULL", i);
            if (r == EA_OK) r = check_address(T.m_scale, EA_T_F32, "m_scale");
            if (r == EA_OK) r = check_address(T.v_scale, EA_T_F32, "v_scale");
        }
        if (T.copy) {
            if (cfg->copy_type != EA_T_BF16 && cfg->copy_type != EA_T_F16)
                return lm_fail(EA_E_INVAL, "copies are bfloat16 or binary16");
            if (r == EA_OK) r = check_address(T.copy, cfg->copy_type, "a copy");
        }
        if (r != EA_OK) return r;
    }
    return EA_OK;
}

struct AdamLayout {
    size_t first, tensors, state;
    size_t total() const { return first + tensors + state; }
};

AdamLayout adam_layout(const ea_adamw_config &cfg)
{
    const size_t n = cfg.n_tensors, launches = (n + kGradBatch - 1) / kGradBatch;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    return {up((n + launches) * 8), up(n * sizeof(ea_adamw_tensor)), up(sizeof(AdamState))};
}

template <class P, class G>
void launch_adamw(const ea_adamw &h, const ea_adamw::Launch &l, const AdamArgs &a, const GradList &list)
{
    const bool half = h.cfg.copy_type == EA_T_F16;
    if (h.cfg.state_bits == 32) {
        if (half) adamw_kernel<P, G, f16, 32><<<l.grid, kAdamThreads, 0, h.stream>>>(a, list);
        else adamw_kernel<P, G, bf16, 32><<<l.grid, kAdamThreads, 0, h.stream>>>(a, list);
    } else {
        if (half) adamw_kernel<P, G, f16, 8><<<l.grid, kAdamThreads, 0, h.stream>>>(a, list);
        else adamw_kernel<P, G, bf16, 8><<<l.grid, kAdamThreads, 0, h.stream>>>(a, list);
    }
}

template <class P>
void launch_adamw(const ea_adamw &h, const ea_adamw::Launch &l, const AdamArgs &a, const GradList &list)
{
    switch (h.cfg.grad_type) {
    case EA_T_F32: launch_adamw<P, float>(h, l, a, list); break;
    case EA_T_BF16: launch_adamw<P, bf16>(h, l, a, list); break;
    default: launch_adamw<P, f16>(h, l, a, list);
    }
}

}  // namespace

extern "C" {

int ea_adamw_workspace_bytes(const ea_adamw_config *cfg, size_t *bytes)
{
    if (!bytes) return lm_fail(EA_E_INVAL, "bytes is NULL");
    const int r = validate(cfg);
    if (r != EA_OK) return r;
    *bytes = adam_layout(*cfg).total();
    return EA_OK;
}

int ea_adamw_init(const ea_adamw_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_adamw **out)
{
    if (!out) return lm_fail(EA_E_INVAL, "out is NULL");
    *out = nullptr;
    int r = validate(cfg);
    if (r != EA_OK) return r;
    const AdamLayout L = adam_layout(*cfg);
    if ((r = check_workspace(workspace, workspace_bytes, L.total())) != EA_OK) return r;
    ea_adamw *h = new (std::nothrow) ea_adamw;
    if (!h) return lm_fail(EA_E_INVAL, "out of host memory");
    r = h->dev.query();
    try {
        h->stream = static_cast<cudaStream_t>(stream);
        h->cfg = *cfg;
        h->cfg.tensors = nullptr;
        h->tensors.assign(cfg->tensors, cfg->tensors + cfg->n_tensors);
        for (int i = 0; i < cfg->n_tensors; i += kGradBatch) {
            ea_adamw::Launch l{i, std::min(kGradBatch, cfg->n_tensors - i), 0, 0, static_cast<int64_t>(h->table.size())};
            for (int k = 0; k < l.n_tensors; ++k) {
                h->table.push_back(l.units);
                l.units += (h->tensors[i + k].size + kBlock - 1) / kBlock;
            }
            h->table.push_back(l.units);
            const int64_t ctas = (l.units + kAdamThreads / 32 - 1) / (kAdamThreads / 32);
            l.grid = static_cast<int>(std::clamp<int64_t>(ctas, 1, h->dev.sms * kAdamCtasPerSm));
            h->launches.push_back(l);
        }
    } catch (const std::bad_alloc &) {
        r = lm_fail(EA_E_INVAL, "out of host memory");
    }
    if (r == EA_OK) {
        char *p = static_cast<char *>(workspace);
        h->d_first = reinterpret_cast<int64_t *>(p);
        h->d_tensors = reinterpret_cast<ea_adamw_tensor *>(p += L.first);
        h->d_state = reinterpret_cast<AdamState *>(p += L.tensors);
        AdamState &s = h->start;
        s.t = cfg->step;
        s.b1 = std::pow(static_cast<double>(cfg->beta1), static_cast<double>(cfg->step + 1));
        s.b2 = std::pow(static_cast<double>(cfg->beta2), static_cast<double>(cfg->step + 1));
        const double root = std::sqrt(1.0 - s.b2);
        s.a = static_cast<float>(root / (1.0 - s.b1));
        s.e = static_cast<float>(cfg->eps * root);
        auto upload = [&](void *dst, const void *src, size_t n) {
            if (r == EA_OK) r = lm_cuda(cudaMemcpyAsync(dst, src, n, cudaMemcpyHostToDevice, h->stream), "table upload");
        };
        upload(h->d_first, h->table.data(), h->table.size() * 8);
        upload(h->d_tensors, h->tensors.data(), h->tensors.size() * sizeof(ea_adamw_tensor));
        upload(h->d_state, &s, sizeof s);
    }
    if (r != EA_OK) {
        delete h;
        return r;
    }
    *out = h;
    return EA_OK;
}

int ea_adamw_step(ea_adamw *h, const void *const *grads, float lr, const float *clip)
{
    if (!h) return lm_fail(EA_E_INVAL, "handle is NULL");
    if (!grads) return lm_fail(EA_E_INVAL, "grads is NULL");
    if (!std::isfinite(lr)) return lm_fail(EA_E_INVAL, "lr must be finite");
    int r = clip ? check_address(clip, EA_T_F32, "clip") : EA_OK;
    for (size_t i = 0; r == EA_OK && i < h->tensors.size(); ++i)
        if (h->tensors[i].size) r = check_address(grads[i], h->cfg.grad_type, "a gradient");
    if (r == EA_OK) r = h->dev.check();
    if (r != EA_OK) return r;
    for (size_t k = 0; k < h->launches.size(); ++k) {
        const ea_adamw::Launch &l = h->launches[k];
        GradList list{};
        std::copy(grads + l.first_tensor, grads + l.first_tensor + l.n_tensors, list.g);
        AdamArgs a{};
        a.units = l.units;
        a.n_tensors = l.n_tensors;
        a.tensor0 = l.first_tensor;
        a.first = h->d_first + l.first_at;
        a.tensors = h->d_tensors + l.first_tensor;
        a.state = h->d_state;
        a.last = k + 1 == h->launches.size();
        a.lr = lr;
        a.beta1 = h->cfg.beta1;
        a.beta2 = h->cfg.beta2;
        a.c1 = 1.0f - h->cfg.beta1;
        a.c2 = 1.0f - h->cfg.beta2;
        a.beta1d = h->cfg.beta1;
        a.beta2d = h->cfg.beta2;
        a.eps = h->cfg.eps;
        a.minus_zero = -0.0f;
        for (uint32_t k = 0; k < 10; ++k)
            a.keys[k] = make_uint2(static_cast<uint32_t>(h->cfg.seed) + k * 0x9E3779B9u, static_cast<uint32_t>(h->cfg.seed >> 32) + k * 0xBB67AE85u);
        a.clip = clip;
        if (h->cfg.param_type == EA_T_F32) launch_adamw<float>(*h, l, a, list);
        else launch_adamw<bf16>(*h, l, a, list);
        if ((r = lm_cuda(cudaGetLastError(), "launch")) != EA_OK) return r;
    }
    return EA_OK;
}

int ea_adamw_step_index(ea_adamw *h, int64_t *t)
{
    if (!h || !t) return lm_fail(EA_E_INVAL, "NULL argument");
    int r = lm_cuda(cudaMemcpyAsync(t, &h->d_state->t, 8, cudaMemcpyDeviceToHost, h->stream), "step read");
    if (r == EA_OK) r = lm_cuda(cudaStreamSynchronize(h->stream), "stream synchronize");
    return r;
}

int ea_adamw_destroy(ea_adamw *h)
{
    delete h;
    return EA_OK;
}

}  // extern "C"
