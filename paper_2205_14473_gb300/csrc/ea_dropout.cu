// ea_dropout.cu -- ea_dropout_apply.
//
// Bound by HBM, with the generator's 60 instructions for eight elements beside it (half of the ALU's slots).  One GB300, us a call,
// GB/s of the bytes that a call cannot do without, against a copy's 6,767:
//   16,384 x 1600 bf16, with a residual   25.3 us, 6,210 GB/s; off a 16-byte boundary 36, without and rows of 1601 in 1611 58
//   65,536 x 1600 bf16, without           68.0 us, 6,170 GB/s
//   260,096 x 768, binary32 to bf16       173.4 us, 6,910 GB/s
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

// One element: x as kept or dropped by its half word, and what is added.
template <class X, class Y>
__device__ __forceinline__ Y drop_one(const DropArgs &a, uint32_t half, X x, const Y *add)
{
    float y = half >= a.limit ? __fmul_rn(to_f32(x), a.scale) : 0.0f;
    if (add) y = __fadd_rn(y, to_f32(*add));
    return from_f32<Y>(y);
}

// Any rows: a warp takes 256 consecutive elements of the call, a lane forms the words of eight of them, and through shared memory every
// lane gets the half words of every 32nd, so that accesses of single elements lie side by side (16,384 x 1600 bf16 with a residual,
// off every boundary, 36 us; 87 with eight consecutive elements a lane).  FLAT: all rows are one.
template <class X, class Y, bool FLAT>
__global__ void __launch_bounds__(kDropThreads) dropout_any_kernel(const DropArgs a, const RowsOf<const X> xs, const RowsOf<const Y> adds, const RowsOf<Y> ys)
{
    __shared__ uint4 words[kDropThreads];
    const int lane = threadIdx.x % 32;
    const uint16_t *halves = reinterpret_cast<const uint16_t *>(words + (threadIdx.x - lane)) + lane;
    const uint2 counter = drop_counter(a);
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kDropThreads / 32);
    for (int64_t base = (static_cast<int64_t>(blockIdx.x) * (kDropThreads / 32) + threadIdx.x / 32) * 256; base < a.n; base += warps * 256) {
        const int left = static_cast<int>(min(a.n - base, int64_t{256})) - lane;  // of element 32 k + lane: there if below it
        X x[8];
        Y add[8], *to[FLAT ? 1 : 8];
        if constexpr (FLAT) {
            to[0] = ys.p + (base + lane);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (32 * k < left) {
                    x[k] = xs.p[base + lane + 32 * k];
                    if (adds.p) add[k] = adds.p[base + lane + 32 * k];
                }
        } else {
            int64_t r = (base + lane) / a.dim, column = base + lane - r * a.dim;
            const X *px = nullptr;
            const Y *padd = nullptr;
            Y *py = nullptr;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if ((k == 0 || column >= a.dim) && 32 * k < left) {  // another row
                    while (column >= a.dim) column -= a.dim, ++r;
                    const uint32_t row = static_cast<uint32_t>(r);
                    px = xs.row(a.rows, row) + column;
                    py = ys.row(a.rows, row) + column;
                    if (adds.p) padd = adds.row(a.rows, row) + column;
                }
                if (32 * k < left) {
                    x[k] = *px;
                    if (adds.p) add[k] = *padd;
                }
                to[k] = py;
                column += 32, px += 32, padd += 32, py += 32;
            }
        }
        words[threadIdx.x] = drop_words(a, base / kDropVec + lane, counter);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (32 * k < left) {
                Y *p = FLAT ? to[0] + 32 * k : to[FLAT ? 0 : k];
                *p = drop_one(a, halves[32 * k], x[k], adds.p ? &add[k] : nullptr);
            }
        __syncwarp();
    }
}

// Eight elements as they lie in memory, in accesses of 16 bytes, or of 32 for binary32.
template <class T>
struct alignas(8 * sizeof(T)) Eight {
    T x[8];
};
__device__ __forceinline__ Eight<float> load_eight(const float *p)
{
    Eight<float> r;
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(r.x[0]), "=f"(r.x[1]), "=f"(r.x[2]), "=f"(r.x[3]), "=f"(r.x[4]), "=f"(r.x[5]), "=f"(r.x[6]), "=f"(r.x[7])
                 : "l"(p)
                 : "memory");
    return r;
}
template <class T>
__device__ __forceinline__ Eight<T> load_eight(const T *p)
{
    return *reinterpret_cast<const Eight<T> *>(p);
}
__device__ __forceinline__ void store_eight(float *p, const float (&x)[8])
{
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]),
                 "f"(x[6]), "f"(x[7])
                 : "memory");
}
__device__ __forceinline__ void store_eight(bf16 *p, const float (&x)[8])
{
    Eight<bf16> r;
#pragma unroll
    for (int i = 0; i < 8; i += 2) *reinterpret_cast<__nv_bfloat162 *>(r.x + i) = __floats2bfloat162_rn(x[i], x[i + 1]);
    *reinterpret_cast<Eight<bf16> *>(p) = r;
}
__device__ __forceinline__ void store_eight(f16 *p, const float (&x)[8])
{
    Eight<f16> r;
#pragma unroll
    for (int i = 0; i < 8; i += 2) *reinterpret_cast<__half2 *>(r.x + i) = __floats2half2_rn(x[i], x[i + 1]);
    *reinterpret_cast<Eight<f16> *>(p) = r;
}

// CTAs of an SM.  Of 16-bit types alone, whose threads have 16 or 32 bytes on their way, as many as fit (16,384 x 1600 with a
// residual 25.4 us; 5 of them 27.0); with binary32 fewer (260,096 x 768 to bf16 174 us; 8 of them 200).
template <class X, class Y>
constexpr int kDropCtas = sizeof(X) + sizeof(Y) == 4 ? 8 : 5;

// Rows that are whole blocks of eight, each on its boundary, `packs` of them a row (0: all in one); limit below 2^16.  The
// random words are formed while the loads are on their way.
template <class X, class Y, bool ADD>
__global__ void __launch_bounds__(kDropThreads, kDropCtas<X, Y>) dropout_packs_kernel(const DropArgs a, const Rows packs, const RowsOf<const X> xs,
                                                                                       const RowsOf<const Y> adds, const RowsOf<Y> ys)
{
    const uint2 counter = drop_counter(a);
    const int64_t blocks = a.n / kDropVec, stride = static_cast<int64_t>(gridDim.x) * kDropThreads;
    const uint32_t limit = a.limit << 16;
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * kDropThreads + threadIdx.x; q < blocks; q += stride) {
        uint32_t r = 0;
        int64_t column = q * kDropVec;
        if (packs.inner) {
            r = packs.outer_of(static_cast<uint32_t>(q));
            column = static_cast<int64_t>(static_cast<uint32_t>(q) - r * packs.inner) * kDropVec;
        }
        const Eight<X> x = load_eight(xs.row(a.rows, r) + column);
        Eight<Y> add;
        if constexpr (ADD) add = load_eight(adds.row(a.rows, r) + column);
        const uint4 w = drop_words(a, q, counter);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool kept = (i & 1 ? word[i >> 1] : word[i >> 1] << 16) >= limit;
            y[i] = kept ? __fmul_rn(to_f32(x.x[i]), a.scale) : 0.0f;
            if constexpr (ADD) y[i] = __fadd_rn(y[i], to_f32(add.x[i]));
        }
        store_eight(ys.row(a.rows, r) + column, y);
    }
}

// The up to seven elements behind the blocks of one row, a thread each (in the kernel above they would cost every thread registers:
// 16,384 x 1600 bf16 35.6 us instead of 25.3).
template <class X, class Y>
__global__ void dropout_tail_kernel(const DropArgs a, const X *x, const Y *add, Y *y)
{
    const int64_t q = a.n / kDropVec, e = q * kDropVec + threadIdx.x;
    if (e >= a.n) return;
    const uint4 w = drop_words(a, q, drop_counter(a));
    const uint32_t word = threadIdx.x < 2 ? w.x : threadIdx.x < 4 ? w.y : threadIdx.x < 6 ? w.z : w.w;
    y[e] = drop_one(a, threadIdx.x & 1 ? word >> 16 : word & 0xffffu, x[e], add ? add + e : nullptr);
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

constexpr int kDropAnyCtas = 4;  // of an SM

// Whether a tensor's rows lie one behind another.
bool follows(const ea_dropout_call *c, int64_t outer, int64_t inner)
{
    return (c->inner <= 1 || inner == c->dim) && (c->outer <= 1 || outer == c->inner * c->dim);
}

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
        // all rows one behind another are one row
        const bool flat = follows(c, c->x_outer, c->x_inner) && follows(c, c->y_outer, c->y_inner) && (!add || follows(c, c->add_outer, c->add_inner));
        const int64_t dim = flat ? a.n / kDropVec * kDropVec : a.dim, outer = flat ? 1 : c->outer, inner = flat ? 1 : c->inner, blocks = over<int64_t>(a.n, kDropVec);
        auto whole = [&](const void *p, int32_t type, int64_t o, int64_t i) { return rows_on(8 * type_bytes(type), p, type, dim, outer, inner, o, i); };
        const bool wide = whole(x, c->x_type, c->x_outer, c->x_inner) && whole(y, c->y_type, c->y_outer, c->y_inner) &&
                          (!add || whole(add, c->y_type, c->add_outer, c->add_inner));
        if (wide && (flat || (blocks < kMaxRows && dim > kDropVec)) && a.limit < 65536) {
            if (flat) a.rows = Rows{};
            const Rows packs = flat ? Rows{} : rows_of(dim / kDropVec);
            const int64_t ctas = std::min<int64_t>(over<int64_t>(a.n / kDropVec, kDropThreads), h->dev.sms * kDropCtas<X, Y>);
            auto kernel = add ? dropout_packs_kernel<X, Y, true> : dropout_packs_kernel<X, Y, false>;
            if (ctas) kernel<<<static_cast<unsigned>(ctas), kDropThreads, 0, h->stream>>>(a, packs, xs, adds, ys);
            if (a.n % kDropVec) dropout_tail_kernel<X, Y><<<1, kDropVec, 0, h->stream>>>(a, xs.p, adds.p, ys.p);
            return;
        }
        if (flat) a.rows = Rows{};
        const int64_t ctas = std::min<int64_t>(over<int64_t>(a.n, 256 * (kDropThreads / 32)), h->dev.sms * kDropAnyCtas);
        auto kernel = flat ? dropout_any_kernel<X, Y, true> : dropout_any_kernel<X, Y, false>;
        kernel<<<static_cast<unsigned>(ctas), kDropThreads, 0, h->stream>>>(a, xs, adds, ys);
    });
    return lm_cuda(cudaGetLastError(), "launch");
}

int ea_dropout_destroy(ea_dropout *h)
{
    delete h;
    return EA_OK;
}

}  // extern "C"
