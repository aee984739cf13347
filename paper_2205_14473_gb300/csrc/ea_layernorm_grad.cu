// ea_layernorm_grad.cu -- ea_layernorm_backward.
//
// The gradients of weight and bias are sums over rows: every thread keeps those of its columns, a CTA's groups are added at its
// end, and a second launch adds the CTAs' in order.
// Bound by a row's chain of dependent steps and HBM together (issue slots 58% used).  One GB300, us a call, GB/s as in ea_layernorm.cu:
//   16,384 x 1600 bf16 with the residual's gradient 39.4 us, 5,320 GB/s; 1601 wide 63;  8,192 x 4,096 48 us, 5,600 GB/s;  4,096 x 8,192 49.6
//   rows that registers do not hold: 4,096 x 12,288 bf16 465 us, 870 GB/s
//   7,021 x 769 binary32 17.6 us, 3,690 GB/s, of which 7 are what 64 rows take: launches, weights and the join
#include "ea_layernorm.cuh"

namespace ea {

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

// The parts' sums added: a CTA takes 32 columns of dw (blockIdx.y = 0) or db, a warp every 32nd part, kJoinAhead of them on their
// way at a time, and then a column's 32 sums.
constexpr int kJoinRows = 32, kJoinAhead = 5;

__global__ void __launch_bounds__(kColumnLanes *kJoinRows) ln_join_kernel(const LnArgs a, const float *partial, int parts, void *dw, void *db, int accumulate)
{
    __shared__ float red[kJoinRows][kColumnLanes + 1];
    const int lane = threadIdx.x % kColumnLanes, row = threadIdx.x / kColumnLanes;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kColumnLanes, column = first + lane;
    void *out = blockIdx.y ? db : dw;
    pdl_wait();
    if (!out) return;
    float s = 0.0f;
    const float *from = partial + blockIdx.y * a.dim + column;
    for (int k = row; k < parts; k += kJoinRows * kJoinAhead) {
        float v[kJoinAhead];
#pragma unroll
        for (int j = 0; j < kJoinAhead; ++j) {
            const int64_t part = k + j * kJoinRows;
            v[j] = part < parts && column < a.dim ? from[part * 2 * a.dim] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kJoinAhead; ++j) s = __fadd_rn(s, v[j]);
    }
    red[row][lane] = s;
    __syncthreads();
    s = warp_sum(red[lane][row]);
    if (lane || first + row >= a.dim) return;
    if (accumulate) s = __fadd_rn(s, load_any(out, a.grad_type, first + row));
    store_any(out, a.grad_type, first + row, s);
}

// One CTA to an SM; groups of G threads walk through the rows, and leave the CTA's sums of dw and db in its part.
template <class X, class Y, int VEC, int G>
__global__ void __launch_bounds__(kBackThreads, 1) ln_backward_kernel(const LnArgs a, const RowsOf<const Y> dys, const RowsOf<const X> xs, const float *stats,
                                                                      const RowsOf<const X> adds, const RowsOf<X> dxs, float *partial)
{
    constexpr int kGroups = kBackThreads / G, W = G / 32, T = kBackThreads, kDepth = kBackDepth<X, Y>;
    pdl_trigger();
    constexpr bool kRing = VEC > 1;
    using HX = Held<X, VEC>;
    using HY = Held<Y, VEC>;
    extern __shared__ __align__(16) unsigned char memory[];
    float *sums = reinterpret_cast<float *>(memory);  // at the end: each group's dw, then its db
    // A stage: packs of x, of dy and of the added rows, one per thread each.
    typename HX::Pack *ring_x = reinterpret_cast<typename HX::Pack *>(memory) + threadIdx.x, *ring_add = ring_x + kDepth * HX::kPacks * T;
    typename HY::Pack *ring_y = reinterpret_cast<typename HY::Pack *>(memory + 2 * sizeof(X) * kHeld * T * kDepth) + threadIdx.x;
    __shared__ float2 parts[2][kBackThreads / 32];
    const int lane = threadIdx.x % G, group = threadIdx.x / G, warp = threadIdx.x / 32;
    const uint32_t stride = gridDim.x * kGroups;
    uint32_t r = blockIdx.x * kGroups + group;
    const int packs = static_cast<int>(a.dim / VEC);
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

extern "C" {

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
            const RowsOf<const X> adds = rows_at<const X>(c, dx ? add : nullptr, c->add_outer, c->add_inner);
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
            RowsLie lie{c, a.dim, kVec};
            lie.add(x, c->x_type, c->x_outer, c->x_inner);
            lie.add(dy, c->y_type, c->y_outer, c->y_inner);
            if (dx) lie.add(dx, c->x_type, c->dx_outer, c->dx_inner);
            if (dx && add) lie.add(add, c->x_type, c->add_outer, c->add_inner);
            if (lie.flat) a.rows = Rows{};
            with_rows<kVec>(a.dim, lie.whole, [&](auto group, auto vec) {
                constexpr int G = decltype(group)::value, V = decltype(vec)::value;
                const uint32_t ctas = std::min<uint32_t>(over<uint32_t>(a.n, kBackThreads / G), h->dev.sms);
                float *partial = dw || db ? h->partial : nullptr;
                if (partial) parts = static_cast<int>(ctas);
                auto kernel = ln_backward_kernel<X, Y, V, G>;
                const size_t ring = V > 1 ? kBackDepth<X, Y> * kBackThreads * kHeld * (2 * sizeof(X) + sizeof(Y)) : kSumsBytes;
                e = h->allowed(kernel, ring);
                if (e == cudaSuccess) kernel<<<ctas, kBackThreads, ring, h->stream>>>(a, dys, xs, stats, adds, dxs, partial);
            });
        }
    });
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess && (dw || db) && !(accumulate && !a.n)) {
        const dim3 grid(static_cast<unsigned>(over<int64_t>(a.dim, kColumnLanes)), 2);
        e = launch_lm(ln_join_kernel, grid, kColumnLanes * kJoinRows, 0, h->stream, a.n != 0, 1, a, static_cast<const float *>(h->partial), parts, dw, db,
                      static_cast<int>(accumulate));
    }
    return lm_cuda(e, "launch");
}

}  // extern "C"
