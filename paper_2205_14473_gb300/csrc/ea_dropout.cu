// ea_dropout.cu -- ea_dropout_apply.
#include "ea_block.cuh"
#include "ea_device.cuh"

namespace ea {

constexpr int kDropThreads = 256;
constexpr int kDropVec = 8;  // elements that share a block of four random words

struct DropArgs {
    int64_t n, dim;
    Rows rows;
    uint32_t limit;  // half words below it drop their element
    float scale;     // 1 / (1 - p)
    uint2 key;
    uint2 counter;
    const uint64_t *device_counter;
};

// The half words of elements 8 q .. 8 q + 7, two per word.
__device__ __forceinline__ uint4 drop_words(const DropArgs &a, int64_t q, uint2 counter)
{
    return philox4x32_10(make_uint4(static_cast<uint32_t>(q), static_cast<uint32_t>(static_cast<uint64_t>(q) >> 32), counter.x, counter.y), a.key);
}

__device__ __forceinline__ uint2 drop_counter(const DropArgs &a)
{
    if (!a.device_counter) return a.counter;
    const uint64_t c = *a.device_counter;
    return make_uint2(static_cast<uint32_t>(c), static_cast<uint32_t>(c >> 32));
}

// Eight consecutive elements of the call at a time, each found for itself.
template <class X, class Y>
__global__ void __launch_bounds__(kDropThreads) dropout_any_kernel(const DropArgs a, const RowsOf<const X> xs, const RowsOf<const Y> adds, const RowsOf<Y> ys)
{
    const uint2 counter = drop_counter(a);
    const int64_t quads = (a.n + kDropVec - 1) / kDropVec;
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * kDropThreads + threadIdx.x; q < quads; q += static_cast<int64_t>(gridDim.x) * kDropThreads) {
        const uint4 w = drop_words(a, q, counter);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
        int64_t r = q * kDropVec / a.dim, column = q * kDropVec - r * a.dim;
#pragma unroll
        for (int i = 0; i < kDropVec; ++i) {
            if (q * kDropVec + i >= a.n) break;
            const uint32_t half = i & 1 ? word[i >> 1] >> 16 : word[i >> 1] & 0xffffu;
            float x = half >= a.limit ? __fmul_rn(to_f32(xs.row(a.rows, static_cast<uint32_t>(r))[column]), a.scale) : 0.0f;
            if (adds.p) x = __fadd_rn(x, to_f32(adds.row(a.rows, static_cast<uint32_t>(r))[column]));
            ys.row(a.rows, static_cast<uint32_t>(r))[column] = from_f32<Y>(x);
            if (++column == a.dim) column = 0, ++r;
        }
    }
}

}  // namespace ea

using namespace ea;

struct ea_dropout {
    DeviceOf dev;
    cudaStream_t stream = nullptr;
    uint32_t limit = 0;
    float scale = 0.0f;
    uint64_t seed = 0;
};

namespace {

int validate(const ea_dropout_config *cfg)
{
    if (!cfg) return lm_fail(EA_E_INVAL, "config is NULL");
    if (!(cfg->p >= 0.0 && cfg->p <= 1.0)) return lm_fail(EA_E_INVAL, "p must be in [0, 1]");
    return EA_OK;
}

}  // namespace

extern "C" {

int ea_dropout_workspace_bytes(const ea_dropout_config *cfg, size_t *bytes)
{
    if (!bytes) return lm_fail(EA_E_INVAL, "bytes is NULL");
    const int r = validate(cfg);
    if (r != EA_OK) return r;
    *bytes = 0;
    return EA_OK;
}

int ea_dropout_init(const ea_dropout_config *cfg, void *, size_t, void *stream, ea_dropout **out)
{
    if (!out) return lm_fail(EA_E_INVAL, "out is NULL");
    *out = nullptr;
    int r = validate(cfg);
    if (r != EA_OK) return r;
    DeviceOf dev;
    if ((r = dev.query()) != EA_OK) return r;
    ea_dropout *h = new (std::nothrow) ea_dropout;
    if (!h) return lm_fail(EA_E_INVAL, "out of host memory");
    h->dev = dev;
    h->stream = static_cast<cudaStream_t>(stream);
    h->limit = static_cast<uint32_t>(std::nearbyint(cfg->p * 65536.0));
    h->scale = h->limit == 65536 ? 0.0f : static_cast<float>(65536.0 / (65536.0 - h->limit));
    h->seed = cfg->seed;
    *out = h;
    return EA_OK;
}

int ea_dropout_apply(ea_dropout *h, const ea_dropout_call *c, const void *x, const void *add, uint64_t counter, const uint64_t *device_counter, void *y)
{
    if (!h) return lm_fail(EA_E_INVAL, "handle is NULL");
    if (!c) return lm_fail(EA_E_INVAL, "call is NULL");
    constexpr int64_t kMost = int64_t{1} << 40;
    if (c->outer < 0 || c->inner < 0 || c->dim < 0 || c->outer > kMaxRows || c->inner > kMaxRows || c->outer * c->inner > kMaxRows || c->dim > kMost ||
        (c->outer * c->inner && c->dim > kMost / (c->outer * c->inner)))
        return lm_fail(EA_E_INVAL, "%lld x %lld rows of %lld: out of range", static_cast<long long>(c->outer), static_cast<long long>(c->inner),
                       static_cast<long long>(c->dim));
    if (!is_float_type(c->x_type)) return lm_fail(EA_E_INVAL, "unknown type %d of x", c->x_type);
    if (!is_float_type(c->y_type)) return lm_fail(EA_E_INVAL, "unknown type %d of y", c->y_type);
    if (c->x_type != c->y_type && c->x_type != EA_T_F32 && c->y_type != EA_T_F32)
        return lm_fail(EA_E_UNSUPPORTED, "x and y of two different types of 16 bits");
    DropArgs a{};
    a.n = c->outer * c->inner * c->dim;
    int r = EA_OK;
    if (a.n) {
        r = check_address(x, c->x_type, "x");
        if (r == EA_OK) r = check_address(y, c->y_type, "y");
        if (r == EA_OK && add) r = check_address(add, c->y_type, "add");
        if (r == EA_OK) r = check_rows_apart(c->outer, c->inner, c->y_outer, c->y_inner, c->dim, "y");
    }
    if (r == EA_OK && reinterpret_cast<uintptr_t>(device_counter) % 8) r = lm_fail(EA_E_ALIGN, "device_counter is not aligned to its 8 bytes");
    if (r == EA_OK) r = h->dev.check();
    if (r != EA_OK || !a.n) return r;
    a.dim = c->dim;
    a.limit = h->limit;
    a.scale = h->scale;
    a.key = make_uint2(static_cast<uint32_t>(h->seed), static_cast<uint32_t>(h->seed >> 32));
    a.counter = make_uint2(static_cast<uint32_t>(counter), static_cast<uint32_t>(counter >> 32));
    a.device_counter = device_counter;
    if (c->inner > 1 && c->outer > 1) a.rows = rows_of(c->inner);
    with_pair(c->x_type, c->y_type, [&](auto *xt, auto *yt) {
        using X = std::remove_reference_t<decltype(*xt)>;
        using Y = std::remove_reference_t<decltype(*yt)>;
        const bool one = c->inner == 1;
        const RowsOf<const X> xs{static_cast<const X *>(x), c->x_outer, one ? c->x_outer : c->x_inner};
        const RowsOf<const Y> adds{static_cast<const Y *>(add), c->add_outer, one ? c->add_outer : c->add_inner};
        const RowsOf<Y> ys{static_cast<Y *>(y), c->y_outer, one ? c->y_outer : c->y_inner};
        const int64_t ctas = over<int64_t>(over<int64_t>(a.n, kDropVec), kDropThreads);
        dropout_any_kernel<X, Y><<<static_cast<unsigned>(std::min<int64_t>(ctas, h->dev.sms * 8)), kDropThreads, 0, h->stream>>>(a, xs, adds, ys);
    });
    return lm_cuda(cudaGetLastError(), "launch");
}

int ea_dropout_destroy(ea_dropout *h)
{
    delete h;
    return EA_OK;
}

}  // extern "C"
