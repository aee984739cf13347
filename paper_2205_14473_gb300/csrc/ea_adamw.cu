// ea_adamw.cu -- ea_adamw_step: one AdamW step (Loshchilov and Hutter; Adam's bias correction folded into the
// step size and epsilon as in the last remark of Kingma and Ba's Section 2) over a list of tensors, with
// moments in binary32 or in 8 bits.
//
// Measured on one GB300 (us a step, GB/s of the bytes that it cannot do without, against a copy's 6,800):
//   354 M binary32 parameters, bfloat16 gradients and copy, 32-bit states  1,506 to 1,540 us, 6,580 GB/s: HBM
//   ResNet-18's 62 tensors, all binary32                                   60 us, 5,440 GB/s: launch and first loads
//   108 M bfloat16 parameters and gradients, 8-bit states                  336 us, 3,250 GB/s: two limits, below
// An 8-bit step is 80 instructions per coordinate at 14 warps per SM: 65% of the issue slots, the ALU 49% busy, DRAM at a
// third of its rate.  Nine of the generator's ten rounds taken out save 45 us.  But the accesses alone, in the same order
// and with the arithmetic taken out, take 334 us too, where each block's two scales are loaded one block ahead and stored
// by themselves: fewer instructions alone would not make it faster.  With eight blocks' scales moved together the accesses
// take 185 us and the whole step 353.
#include <cuda_fp8.h>

#include <type_traits>

#include "ea_async.cuh"
#include "ea_lm.cuh"

namespace ea {

constexpr int kAdamThreads = 128;
constexpr int kAdamCtasPerSm = 4;  // 128 registers per thread; a persistent grid of them
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

// Within 2^-23 relative of the reciprocal of a normal number (0 for one above 2^126).  With a correctly rounded quotient
// instead, 8-bit steps of 40 M coordinates take 141 us for 130, 32-bit ones of ResNet-18 61.3 for 59.9.
__device__ __forceinline__ float recip_normal(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

constexpr uint32_t kLiftBelow = (127u + 60u) << 23;  // 2^60: the values that sqrt_lifted is used for

// The square roots of 2^64 v for two v, zero or at least 2^-149, rounded to nearest: from y ~ 1 / sqrt(x), the
// remainder x - g^2 of g = x y, exact in a fused operation, corrects g to its last bit (Markstein, "Computation of
// elementary functions on the IBM RISC System/6000 processor", 1990; without the refinement of y and g that the paper
// has in between).  Equal to sqrtf, times 2^32, for every v below 2^60 (ea_adamw_selftest_sqrt).
// It is a third of the call's instructions, and no branch stands between a lane's coordinates.
__device__ __forceinline__ F2 sqrt_lifted(F2 v, F2 none)
{
    float xa, xb, ya, yb;
    const F2 x = fma2(v, both(0x1p64f), none), minus_x = fma2(v, both(-0x1p64f), none);
    unpack2(fma2(v, both(0x1p64f), both(0x1p-100f)), xa, xb);  // not zero
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(ya) : "f"(xa));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(yb) : "f"(xb));
    const F2 y = pack2(ya, yb), g = fma2(x, y, none);
    return fma2(fma2(g, g, minus_x), fma2(y, both(-0.5f), none), g);
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

// Those from p on below n; the others are 0.
template <class T>
__device__ __forceinline__ Quad<T> load_quad(const T *p, int n)
{
    Quad<T> q{};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) q.x[i] = p[i];
    return q;
}
// Those from p on, where `whole`, else the ones below n.
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
    F2 factor, beta1, beta2, c1, c2, e, step, rate;
    F2 none;  // (-0, -0)

    // m <- mb m + c1 g and v <- vb v + c2 g^2 with g the gradient times the factor.
    __device__ __forceinline__ void moments(F2 &m, F2 &v, F2 grad, F2 mb, F2 vb) const
    {
        const F2 g = mul2(grad, factor, none);
        m = add2(mul2(m, mb, none), mul2(g, c1, none));
        v = add2(mul2(v, vb, none), mul2(mul2(g, g, none), c2, none));
    }

    // The new parameters, from the moments and the second one's root (times `unit`, a power of two).
    __device__ __forceinline__ F2 params(F2 p, F2 m, F2 root, F2 unit) const
    {
        float a, b;
        unpack2(fma2(root, unit, e), a, b);
        const F2 q = mul2(m, pack2(recip_normal(a), recip_normal(b)), none);
        return fma2(fma2(q, step, mul2(p, rate, none)), both(-1.0f), p);
    }
};

__device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x); }

// max(|a|, |b|), NaN if either is.
__device__ __forceinline__ float max_magnitude(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}

// Codes of four values x with |x| <= 448 in e4m3, the magnitudes rounded up with the probability of the remainder
// (word: random bits, the low half's or, HIGH, the high half's).
//   normal numbers: the code is the float's exponent and first three mantissa bits, re-biased: with the 20 bits
//     below at the top of a register's lower 24, 16 random bits are added there and the carry does the rounding --
//     one byte permutation, which also brings in the bias, and one multiply-add per value.  The sign is shifted out;
//   below 2^-6 the grid's spacing is 2^-9 throughout: taken value by value, where there is one.
// CLAMP: a value that is not zero does not become zero.
template <bool HIGH, bool CLAMP>
__device__ __forceinline__ uint32_t e4m3_round(const float (&x)[4], const uint32_t (&word)[4], bool finite)
{
    uint32_t t[4];
    const float least = fminf(fminf(fabsf(x[0]), fabsf(x[1])), fminf(fabsf(x[2]), fabsf(x[3])));
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = bits(x[i]) * 16u + __byte_perm(word[i], 0x00400000u, HIGH ? 0x6324 : 0x6104);
    if (least < 0x1p-6f || !finite) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float y = fabsf(x[i]);
            if (y < 0x1p-6f) {
                const float r = static_cast<float>(HIGH ? word[i] >> 16 : word[i] & 0xffffu);
                const float up = __fmaf_rn(r, 0x1p-16f, __fmul_rn(y, 512.0f));
                const uint32_t n = static_cast<uint32_t>(__float2int_rd(up));
                t[i] = (CLAMP && y > 0.0f ? max(n, 1u) : n) << 24;
            } else if (!(y < __int_as_float(0x7f800000))) {
                t[i] = 0x7f000000u;
            }
        }
    }
    uint32_t codes = __byte_perm(__byte_perm(t[0], t[1], 0x0073), __byte_perm(t[2], t[3], 0x0073), 0x5410);
    if (!CLAMP) {  // signed values
        const uint32_t signs = __byte_perm(__byte_perm(bits(x[0]), bits(x[1]), 0x0073), __byte_perm(bits(x[2]), bits(x[3]), 0x0073), 0x5410);
        codes |= signs & 0x80808080u;
    }
    return codes;
}

// 8-bit states are handled as bytes, 32-bit ones as numbers.
template <int BITS>
using AdamCell = typename std::conditional<BITS == 32, float, uint8_t>::type;

// Addresses of this lane's first coordinate in a block, and of the block's scales.
template <class P, class G, class C, class S>
struct AdamPlace {
    P *p;
    const G *g;
    C *copy;
    S *m, *v;
    float *ms, *vs;
    __device__ __forceinline__ void advance(int blocks)
    {
        p += blocks * kBlock;
        g += blocks * kBlock;
        if (copy) copy += blocks * kBlock;
        m += blocks * kBlock;
        v += blocks * kBlock;
        ms += blocks;
        vs += blocks;
    }
};

// What a lane reads of a block: 4 coordinates in each half.
template <class P, class G, class S>
struct AdamBlock {
    Quad<P> p[2];
    Quad<G> g[2];
    Quad<S> m[2], v[2];
};

// A stage of a warp's ring in shared memory: a block, laid out so that a lane copies in, and reads back, its own
// quads alone (no synchronisation between lanes) and the warp's accesses are contiguous.
template <class P, class G, class S>
struct AdamStage {
    Quad<P> p[2][32];
    Quad<G> g[2][32];
    Quad<S> m[2][32], v[2][32];
};

template <class T>
__device__ __forceinline__ void copy_quad(Quad<T> *to, const T *from)
{
    if constexpr (sizeof(T) == 4) cp_async16(to, from);
    else if constexpr (sizeof(T) == 2) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_addr(to)), "l"(from) : "memory");
    else cp_async4(to, from);
}

// The copies of a whole, aligned block, `ahead` blocks from `at`, into a stage.
template <class P, class G, class C, class S>
__device__ __forceinline__ void adam_fetch(const AdamPlace<P, G, C, S> &at, int ahead, AdamStage<P, G, S> &st)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int off = ahead * kBlock + 128 * h;
        copy_quad(&st.p[h][lane], at.p + off);
        copy_quad(&st.g[h][lane], at.g + off);
        copy_quad(&st.m[h][lane], static_cast<const S *>(at.m) + off);
        copy_quad(&st.v[h][lane], static_cast<const S *>(at.v) + off);
    }
}

template <class P, class G, class S>
__device__ __forceinline__ AdamBlock<P, G, S> adam_read(const AdamStage<P, G, S> &st)
{
    const int lane = threadIdx.x & 31;
    AdamBlock<P, G, S> b;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        b.p[h] = st.p[h][lane];
        b.g[h] = st.g[h][lane];
        b.m[h] = st.m[h][lane];
        b.v[h] = st.v[h][lane];
    }
    return b;
}

// n coordinates of a block, from this lane's first on.
template <class P, class G, class C, class S>
__device__ __forceinline__ void adam_load(const AdamPlace<P, G, C, S> &at, int n, AdamBlock<P, G, S> &b)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        b.p[h] = load_quad(at.p + 128 * h, n - 128 * h);
        b.g[h] = load_quad(at.g + 128 * h, n - 128 * h);
        b.m[h] = load_quad(at.m + 128 * h, n - 128 * h);
        b.v[h] = load_quad(at.v + 128 * h, n - 128 * h);
    }
}

// WHOLE: a whole block whose addresses are all aligned to four elements.
template <bool WHOLE, class P, class G, class C, class S>
__device__ __forceinline__ void adam_store(const AdamPlace<P, G, C, S> &at, int n, int h, const float (&p)[4], const Quad<S> &m, const Quad<S> &v)
{
    store_quad(at.p + 128 * h, n - 128 * h, WHOLE, quad_of<P>(p));
    if (at.copy) store_quad(at.copy + 128 * h, n - 128 * h, WHOLE, quad_of<C>(p));
    store_quad(at.m + 128 * h, n - 128 * h, WHOLE, m);
    store_quad(at.v + 128 * h, n - 128 * h, WHOLE, v);
}

// The 32-bit step of a block.
template <bool WHOLE, class P, class G, class C>
__device__ __forceinline__ void adam_block(const AdamArgs &, const AdamStep &s, const AdamPlace<P, G, C, float> &at, int n,
                                           const AdamBlock<P, G, float> &b, float, float, uint64_t, uint32_t, uint32_t)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float p[4], m[4], v[4], g[4];
        quad_values(b.p[h], p);
        quad_values(b.g[h], g);
        quad_values(b.m[h], m);
        quad_values(b.v[h], v);
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            F2 m2 = pack2(m[i], m[i + 1]), v2 = pack2(v[i], v[i + 1]);
            s.moments(m2, v2, pack2(g[i], g[i + 1]), s.beta1, s.beta2);
            unpack2(m2, m[i], m[i + 1]);
            unpack2(v2, v[i], v[i + 1]);
            const F2 root = pack2(__fsqrt_rn(v[i]), __fsqrt_rn(v[i + 1]));
            unpack2(s.params(pack2(p[i], p[i + 1]), m2, root, both(1.0f)), p[i], p[i + 1]);
        }
        adam_store<WHOLE>(at, n, h, p, quad_of<float>(m), quad_of<float>(v));
    }
}

// The 8-bit step of a block.  quad: its first group of four coordinates of this lane, within the tensor.
template <bool WHOLE, class P, class G, class C>
__device__ __forceinline__ void adam_block(const AdamArgs &a, const AdamStep &s, const AdamPlace<P, G, C, uint8_t> &at, int n,
                                           const AdamBlock<P, G, uint8_t> &b, float ms, float vs, uint64_t quad, uint32_t tensor,
                                           uint32_t t)
{
    F2 m[4], v[4];
    // beta1 m scale and beta2 (r scale)^2 are one multiplication each where the power of two leaves the product
    // normal: a scale below 2^-40 goes into the values first
    const bool small = ms < 0x1p-40f || vs < 0x1p-40f;
    const F2 mb = small ? s.beta1 : mul2(s.beta1, both(ms), s.none);
    const F2 vb = small ? s.beta2 : mul2(s.beta2, mul2(both(vs), both(vs), s.none), s.none);
    float am = 0.0f, av = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float mx[4], vx[4], g[4];
        e4m3_values(*reinterpret_cast<const uint32_t *>(&b.m[h]), mx);
        e4m3_values(*reinterpret_cast<const uint32_t *>(&b.v[h]), vx);
        quad_values(b.g[h], g);
        if (small)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                mx[i] = __fmul_rn(mx[i], ms);
                vx[i] = __fmul_rn(vx[i], vs);
            }
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            F2 &m2 = m[2 * h + i / 2], &v2 = v[2 * h + i / 2];
            m2 = pack2(mx[i], mx[i + 1]);
            v2 = pack2(vx[i], vx[i + 1]);
            v2 = mul2(v2, v2, s.none);
            s.moments(m2, v2, pack2(g[i], g[i + 1]), mb, vb);
            float x, y;
            unpack2(m2, x, y);
            am = max_magnitude(max_magnitude(am, x), y);
            unpack2(v2, x, y);
            av = max_magnitude(max_magnitude(av, x), y);
        }
    }
    uint32_t mmax = __reduce_max_sync(0xffffffffu, bits(am)), vmax = __reduce_max_sync(0xffffffffu, bits(av));
    const bool finite = max(mmax, vmax) < 0x7f800000u;
    if (!finite) {  // the scales go by the finite values; the others are held as NaN
        mmax = vmax = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x, y;
            unpack2(m[i], x, y);
            mmax = max(mmax, max(finite_magnitude(x), finite_magnitude(y)));
            unpack2(v[i], x, y);
            vmax = max(vmax, max(finite_magnitude(x), finite_magnitude(y)));
        }
        mmax = __reduce_max_sync(0xffffffffu, mmax);
        vmax = __reduce_max_sync(0xffffffffu, vmax);
    }
    // roots are taken 2^32 times as large, so that subnormal values have one, where none overflows
    const bool lift = finite && vmax < kLiftBelow;
    const F2 unit = both(lift ? 0x1p-32f : 1.0f);
    const int km = scale_exponent(mmax), kv = scale_exponent(bits(__fsqrt_rn(__uint_as_float(vmax))));
    const F2 im = both(power_of_two(-km)), iv = mul2(both(power_of_two(-kv)), unit, s.none);
    if ((threadIdx.x & 31) == 0) {
        *at.ms = power_of_two(km);
        *at.vs = power_of_two(kv);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float p[4], ym[4], yv[4];
        quad_values(b.p[h], p);
        const uint64_t q = quad + 32 * h;
        const uint4 w = philox_words(make_uint4(static_cast<uint32_t>(q), static_cast<uint32_t>(q >> 32), tensor, t), a.keys);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const F2 m2 = m[2 * h + i / 2], v2 = v[2 * h + i / 2];
            F2 root;
            if (lift) {
                root = sqrt_lifted(v2, s.none);
            } else {
                float x, y;
                unpack2(v2, x, y);
                root = pack2(__fsqrt_rn(x), __fsqrt_rn(y));
            }
            unpack2(s.params(pack2(p[i], p[i + 1]), m2, root, unit), p[i], p[i + 1]);
            unpack2(mul2(m2, im, s.none), ym[i], ym[i + 1]);
            unpack2(mul2(root, iv, s.none), yv[i], yv[i + 1]);
        }
        Quad<uint8_t> mq, vq;
        *reinterpret_cast<uint32_t *>(&mq) = mmax || !finite ? e4m3_round<false, false>(ym, word, finite) : 0;
        *reinterpret_cast<uint32_t *>(&vq) = vmax || !finite ? e4m3_round<true, true>(yv, word, finite) : 0;
        adam_store<WHOLE>(at, n, h, p, mq, vq);
    }
}

// A CTA takes a contiguous piece of the launch's blocks of 256 coordinates, its warps in turn: every CTA has the same
// number of blocks but for one, and a warp goes along a tensor with its addresses in registers.  A lane holds four
// consecutive coordinates in each half of a block: every access of the warp is one contiguous piece, and the block's
// scale is one warp reduction.  Whole aligned blocks come through a ring of kAdamStages stages per warp in shared
// memory, filled by asynchronous copies: the loads in flight take no registers, which the arithmetic of the 8-bit
// states needs, and enough of them are in flight to cover their latency.
// Stages: up to 4, in a quarter of an SM's shared memory.
template <class Stage>
constexpr int kAdamStages = std::min(4, 54 * 1024 / (static_cast<int>(sizeof(Stage)) * (kAdamThreads / 32)));

template <class P, class G, class C, int BITS>
__global__ void __launch_bounds__(kAdamThreads, kAdamCtasPerSm)
    adamw_kernel(const __grid_constant__ AdamArgs a, const __grid_constant__ GradList list)
{
    using S = AdamCell<BITS>;
    using Stage = AdamStage<P, G, S>;
    constexpr int kWarps = kAdamThreads / 32, kStages = kAdamStages<Stage>;
    extern __shared__ __align__(16) unsigned char smem[];
    const float factor = a.clip ? a.clip[1] : 1.0f;
    const AdamState st = *a.state;
    const int64_t begin = a.units * blockIdx.x / gridDim.x, end = a.units * (blockIdx.x + 1) / gridDim.x;
    if (!isnan(factor) && begin < end) {
        const int warp = threadIdx.x >> 5, lane4 = (threadIdx.x & 31) * 4;
        Stage *ring = reinterpret_cast<Stage *>(smem) + warp * kStages;
        AdamStep s{both(factor), both(a.beta1), both(a.beta2), both(a.c1), both(a.c2), both(st.e), F2{}, F2{}, both(a.minus_zero)};
        for (int i = tensor_of(a.first, a.n_tensors, begin, 0); i < a.n_tensors; ++i) {
            const int64_t first = a.first[i], lo = max(begin, first), hi = min(end, a.first[i + 1]);
            if (first >= end) break;
            int64_t u = lo + ((warp - (lo - begin)) & (kWarps - 1));  // this warp's next block
            if (u >= hi) continue;
            const ea_adamw_tensor &T = a.tensors[i];
            const int64_t size = T.size, off = (u - first) * kBlock + lane4;
            const float lr = __fmul_rn(a.lr, T.lr_scale);
            s.step = both(__fmul_rn(lr, st.a));
            s.rate = both(__fmul_rn(lr, T.weight_decay));
            AdamPlace<P, G, C, S> at{static_cast<P *>(T.param) + off, static_cast<const G *>(list.g[i]) + off,
                                     T.copy ? static_cast<C *>(T.copy) + off : nullptr, static_cast<S *>(T.m) + off,
                                     static_cast<S *>(T.v) + off, T.m_scale + (u - first), T.v_scale + (u - first)};
            const uint32_t tensor = static_cast<uint32_t>(a.tensor0 + i), t = static_cast<uint32_t>(st.t);
            uint64_t quad = static_cast<uint64_t>(off) >> 2;
            const bool aligned = reinterpret_cast<uintptr_t>(at.p) % sizeof(Quad<P>) == 0 &&
                                 reinterpret_cast<uintptr_t>(at.g) % sizeof(Quad<G>) == 0 &&
                                 reinterpret_cast<uintptr_t>(at.copy) % sizeof(Quad<C>) == 0 &&
                                 (reinterpret_cast<uintptr_t>(at.m) | reinterpret_cast<uintptr_t>(at.v)) % sizeof(Quad<S>) == 0;
            const int64_t whole = aligned ? min(hi, first + size / kBlock) : u;  // blocks below it are whole and aligned
            float ms = 0.0f, vs = 0.0f;
            if (u < whole) {
                if (BITS == 8) {
                    ms = *at.ms;
                    vs = *at.vs;
                }
#pragma unroll
                for (int k = 0; k < kStages - 1; ++k) {
                    if (u + k * kWarps < whole) adam_fetch(at, k * kWarps, ring[k]);
                    cp_async_commit();
                }
                int in = kStages - 1, out = 0;
                for (; u < whole; u += kWarps) {
                    if (u + (kStages - 1) * kWarps < whole) adam_fetch(at, (kStages - 1) * kWarps, ring[in]);
                    cp_async_commit();
                    cp_async_wait<kStages - 1>();
                    const AdamBlock<P, G, S> b = adam_read(ring[out]);
                    const float ms_now = ms, vs_now = vs;
                    if (BITS == 8 && u + kWarps < whole) {
                        ms = at.ms[kWarps];
                        vs = at.vs[kWarps];
                    }
                    adam_block<true>(a, s, at, kBlock, b, ms_now, vs_now, quad, tensor, t);
                    at.advance(kWarps);
                    quad += kWarps * kBlock / 4;
                    in = in + 1 == kStages ? 0 : in + 1;
                    out = out + 1 == kStages ? 0 : out + 1;
                }
            }
            for (; u < hi; u += kWarps) {
                const int n = static_cast<int>(min(size - (u - first) * kBlock, static_cast<int64_t>(kBlock))) - lane4;
                AdamBlock<P, G, S> b;
                adam_load(at, n, b);
                if (BITS == 8) {
                    ms = *at.ms;
                    vs = *at.vs;
                }
                adam_block<false>(a, s, at, n, b, ms, vs, quad, tensor, t);
                at.advance(kWarps);
                quad += kWarps * kBlock / 4;
            }
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

// Counts the v in [0, 2^kLiftBelow) whose sqrt_lifted is not sqrtf's result times 2^32: all of them, two at a time.
constexpr int kSqrtCtas = 152 * 8, kSqrtThreads = 256;
__global__ void __launch_bounds__(kSqrtThreads) sqrt_selftest_kernel(float minus_zero, unsigned long long *unequal)
{
    unsigned long long bad = 0;
    for (uint32_t i = (blockIdx.x * kSqrtThreads + threadIdx.x) * 2; i < kLiftBelow; i += gridDim.x * kSqrtThreads * 2) {
        const float v[2] = {__uint_as_float(i), __uint_as_float(i + 1)};
        float root[2];
        unpack2(sqrt_lifted(pack2(v[0], v[1]), both(minus_zero)), root[0], root[1]);
        for (int k = 0; k < 2; ++k) bad += bits(root[k]) != bits(__fmul_rn(__fsqrt_rn(v[k]), 0x1p32f));
    }
    if (bad) atomicAdd(unequal, bad);
}
__device__ unsigned long long g_sqrt_unequal;

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
    void (*kernel)(AdamArgs, GradList) = nullptr;
    size_t smem = 0;
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

using AdamKernel = void (*)(AdamArgs, GradList);

// The kernel for a configuration's types, and the bytes of its ring.
template <class P, class G, class C, int BITS>
void adam_kernel(AdamKernel &f, size_t &smem)
{
    f = adamw_kernel<P, G, C, BITS>;
    using Stage = AdamStage<P, G, AdamCell<BITS>>;
    smem = sizeof(Stage) * kAdamStages<Stage> * (kAdamThreads / 32);
}
template <class P, class G>
void adam_kernel(const ea_adamw_config &c, AdamKernel &f, size_t &smem)
{
    const bool half = c.copy_type == EA_T_F16;
    if (c.state_bits == 32) half ? adam_kernel<P, G, f16, 32>(f, smem) : adam_kernel<P, G, bf16, 32>(f, smem);
    else half ? adam_kernel<P, G, f16, 8>(f, smem) : adam_kernel<P, G, bf16, 8>(f, smem);
}
template <class P>
void adam_kernel(const ea_adamw_config &c, AdamKernel &f, size_t &smem)
{
    if (c.grad_type == EA_T_F32) adam_kernel<P, float>(c, f, smem);
    else if (c.grad_type == EA_T_BF16) adam_kernel<P, bf16>(c, f, smem);
    else adam_kernel<P, f16>(c, f, smem);
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
    DeviceOf dev;
    if ((r = dev.query()) != EA_OK) return r;
    ea_adamw *h = new (std::nothrow) ea_adamw;
    if (!h) return lm_fail(EA_E_INVAL, "out of host memory");
    h->dev = dev;
    if (cfg->param_type == EA_T_F32) adam_kernel<float>(*cfg, h->kernel, h->smem);
    else adam_kernel<bf16>(*cfg, h->kernel, h->smem);
    r = lm_cuda(cudaFuncSetAttribute(h->kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(h->smem)), "shared memory");
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
        if ((r = lm_cuda(launch_lm(h->kernel, dim3(l.grid), kAdamThreads, h->smem, h->stream, false, 1, a, list), "launch")) != EA_OK) return r;
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

int ea_adamw_selftest_sqrt(void *stream, uint64_t *unequal)
{
    if (!unequal) return lm_fail(EA_E_INVAL, "unequal is NULL");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const unsigned long long zero = 0;
    unsigned long long n = 0;
    void *at = nullptr;
    int r = lm_cuda(cudaGetSymbolAddress(&at, g_sqrt_unequal), "counter");
    if (r == EA_OK) r = lm_cuda(cudaMemcpyAsync(at, &zero, sizeof zero, cudaMemcpyHostToDevice, s), "counter clear");
    if (r == EA_OK) {
        sqrt_selftest_kernel<<<kSqrtCtas, kSqrtThreads, 0, s>>>(-0.0f, static_cast<unsigned long long *>(at));
        r = lm_cuda(cudaGetLastError(), "launch");
    }
    if (r == EA_OK) r = lm_cuda(cudaMemcpyAsync(&n, at, sizeof n, cudaMemcpyDeviceToHost, s), "counter read");
    if (r == EA_OK) r = lm_cuda(cudaStreamSynchronize(s), "stream synchronize");
    if (r == EA_OK) *unequal = n;
    return r;
}

int ea_adamw_destroy(ea_adamw *h)
{
    delete h;
    return EA_OK;
}

}  // extern "C"
