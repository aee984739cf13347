// ea_layernorm.cu -- ea_layernorm_forward and ea_layernorm_backward.
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

// The parts' sums added in order, each thread a column of dw or db.
__global__ void __launch_bounds__(kColumnLanes *kColumnRows) ln_join_kernel(const LnArgs a, const float *partial, int parts, void *dw, void *db, int accumulate)
{
    __shared__ float red[kColumnRows][kColumnLanes];
    void *out = blockIdx.y ? db : dw;
    if (!out) return;
    const int64_t column = static_cast<int64_t>(blockIdx.x) * kColumnLanes + threadIdx.x;
    float s = 0.0f;
    if (column < a.dim)
        for (int k = threadIdx.y; k < parts; k += kColumnRows) s = __fadd_rn(s, partial[(static_cast<int64_t>(k) * 2 + blockIdx.y) * a.dim + column]);
    red[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y || column >= a.dim) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < kColumnRows; ++i) s = __fadd_rn(s, red[i][threadIdx.x]);
    if (accumulate) s = __fadd_rn(s, load_any(out, a.grad_type, column));
    store_any(out, a.grad_type, column, s);
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
int64_t max_parts(const ea_layernorm_config &c)
{
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
    with_pair(c->x_type, c->y_type, [&](auto *xt, auto *yt) {
        using X = std::remove_reference_t<decltype(*xt)>;
        using Y = std::remove_reference_t<decltype(*yt)>;
        if constexpr (std::is_same<X, Y>::value || std::is_same<X, float>::value) {
            const unsigned grid = std::min<unsigned>(a.n, h->dev.sms * 8);
            ln_forward_any_kernel<X, Y><<<grid, kNormRowThreads, 0, h->stream>>>(a, rows_at<const X>(c, x, c->x_outer, c->x_inner),
                                                                                 rows_at<Y>(c, y, c->y_outer, c->y_inner), stats);
        }
    });
    return lm_cuda(cudaGetLastError(), "launch");
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
    with_pair(c->x_type, c->y_type, [&](auto *xt, auto *yt) {
        using X = std::remove_reference_t<decltype(*xt)>;
        using Y = std::remove_reference_t<decltype(*yt)>;
        if constexpr (std::is_same<X, Y>::value || std::is_same<X, float>::value) {
            if (!a.n) return;
            const RowsOf<const Y> dys = rows_at<const Y>(c, dy, c->y_outer, c->y_inner);
            const RowsOf<const X> xs = rows_at<const X>(c, x, c->x_outer, c->x_inner);
            if (dw || db) {  // before dx, which may be in the place of dy or x
                const int64_t most = max_parts(h->cfg), part = over<int64_t>(over<int64_t>(a.n, most), kColumnRows) * kColumnRows;
                parts = static_cast<int>(over<int64_t>(a.n, part));
                const dim3 grid(static_cast<unsigned>(over<int64_t>(a.dim, kColumnLanes)), parts);
                ln_columns_any_kernel<X, Y><<<grid, dim3(kColumnLanes, kColumnRows), 0, h->stream>>>(a, dys, xs, stats, static_cast<uint32_t>(part), h->partial);
            }
            if (dx)
                ln_dx_any_kernel<X, Y><<<std::min<unsigned>(a.n, h->dev.sms * 8), kNormRowThreads, 0, h->stream>>>(
                    a, dys, xs, stats, rows_at<const X>(c, add, c->add_outer, c->add_inner), rows_at<X>(c, dx, c->dx_outer, c->dx_inner));
        }
    });
    if ((r = lm_cuda(cudaGetLastError(), "launch")) != EA_OK) return r;
    if ((dw || db) && !(accumulate && !a.n)) {
        const dim3 grid(static_cast<unsigned>(over<int64_t>(a.dim, kColumnLanes)), 2);
        ln_join_kernel<<<grid, dim3(kColumnLanes, kColumnRows), 0, h->stream>>>(a, h->partial, parts, dw, db, accumulate);
    }
    return lm_cuda(cudaGetLastError(), "launch");
}

int ea_layernorm_destroy(ea_layernorm *h)
{
    delete h;
    return EA_OK;
}

}  // extern "C"
