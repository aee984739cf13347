// ea_layernorm.cu -- ea_layernorm_forward.
//
// Mean and variance: each warp's mean and the squares about it, joined (Chan, Golub and LeVeque, "Updating formulae and a
// pairwise algorithm for computing sample variances"), so that the variance does not cancel and a row costs one barrier.
// Bound by a row's chain of dependent steps (two reductions by shuffles and a barrier one behind another, one row at a time in a CTA:
// issue slots 60% used by 28 warps an SM, 194 instructions for a warp's part of a row) where rows are whole 16-byte packs, else
// by accesses of single elements.  One GB300, us a call, GB/s of the bytes that a call cannot do without, against a copy's 6,767:
//   16,384 x 1600 bf16 21.5 us, 4,900 GB/s; 1601 wide 28.5;  262,144 x 128 23.7 us, 5,760 GB/s;  8,192 x 4,096 26 us, 5,170 GB/s
//   16,384 x 1600, binary32 to bf16 27 us, 5,800 GB/s;  4,096 x 8,192 bf16 33.7 us, 3,990 GB/s, one CTA to an SM
//   rows that registers do not hold, read three times by single elements: 4,096 x 12,288 bf16 161 us, 1,250 GB/s
#include "ea_layernorm.cuh"

namespace ea {

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

// A CTA is a group of warps, or 128 threads of smaller groups.
template <int G>
constexpr int kForwardCta = G > 32 ? G : 128;

// Threads of an SM, all of them resident: what registers allow of the kernel at hand (16,384 x 1600 bf16 21.5 us; with 768 22.2,
// with 1,024, a few of whose CTAs wait for the others to end, 26).
template <int VEC>
constexpr int kForwardThreads = VEC == 1 ? 640 : 896;

template <class X, class Y, int VEC, int G>
__global__ void __launch_bounds__(kForwardCta<G>, kForwardThreads<VEC> / kForwardCta<G>) ln_forward_kernel(const LnArgs a, const RowsOf<const X> xs, const RowsOf<Y> ys, float *stats)
{
    constexpr int kThreads = kForwardCta<G>, kGroups = kThreads / G, W = G / 32, kDepth = kForwardDepth;
    constexpr bool kRing = VEC > 1;
    using H = Held<X, VEC>;
    using Pack = typename H::Pack;
    extern __shared__ __align__(16) unsigned char memory[];
    Pack *ring = reinterpret_cast<Pack *>(memory) + threadIdx.x;  // a stage: kPacks, one per thread each
    __shared__ float2 parts[2][W > 1 ? W : 1];  // each warp's mean and squares about it, of this row and the last
    __shared__ float share[W > 1 ? W : 1], counts[W > 1 ? W : 1];  // each warp's elements, and their share of the row's
    const int lane = threadIdx.x % G, warp = threadIdx.x / 32;
    const uint32_t stride = gridDim.x * kGroups;
    uint32_t r = blockIdx.x * kGroups + threadIdx.x / G;
    const int packs = static_cast<int>(a.dim / VEC);
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
        for (int k = 0; k < kHeld / VEC; ++k) {
            const int from = (first + k * G) * VEC, to = from + (G < 32 ? G : 32) * VEC;
            n += max(min(to, static_cast<int>(a.dim)) - from, 0);
        }
        return n;
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
        const float rstd = rsqrt_of(__fmaf_rn(squares, a.inverse, a.eps));
        const F2 scale = both(rstd);
#pragma unroll
        for (int i = 0; i < kHeld / 2; ++i) x[i] = fma2(times2(add2(x[i], minus), scale), w[i], b[i]);
        if (r < a.n) {
            Held<Y, VEC>::template store<G>(ys.row(a.rows, r), lane, packs, x);
            if (stats && lane == 0) *reinterpret_cast<float2 *>(stats + 2 * static_cast<int64_t>(r)) = make_float2(mean, rstd);
        }
    }
}

}  // namespace ea

using namespace ea;

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
            RowsLie lie{c, a.dim, kVec};
            lie.add(x, c->x_type, c->x_outer, c->x_inner);
            lie.add(y, c->y_type, c->y_outer, c->y_inner);
            if (lie.flat) a.rows = Rows{};
            with_rows<kVec>(a.dim, lie.whole, [&](auto group, auto vec) {
                constexpr int G = decltype(group)::value, V = decltype(vec)::value, kThreads = kForwardCta<G>;
                const uint32_t ctas = over<uint32_t>(a.n, kThreads / G), most = h->dev.sms * (kForwardThreads<V> / kThreads);
                auto kernel = ln_forward_kernel<X, Y, V, G>;
                const size_t ring = V > 1 ? kForwardDepth * kThreads * kHeld * sizeof(X) : 0;
                e = h->allowed(kernel, ring);
                if (e == cudaSuccess) kernel<<<std::min(ctas, most), kThreads, ring, h->stream>>>(a, xs, ys, stats);
            });
        }
    });
    return lm_cuda(e == cudaSuccess ? cudaGetLastError() : e, "launch");
}

int ea_layernorm_destroy(ea_layernorm *h)
{
    delete h;
    return EA_OK;
}

}  // extern "C"
