// ea_norm.cu -- ea_grad_norm: the 2-norm of a list of gradients and the factor that clips them.
//
// One launch for up to kGradBatch tensors.  108 M bfloat16 values take 39.8 us (5,450 GB/s of a copy's 6,800), 62
// tensors of 11.7 M binary32 values 16.4 us (2,850 GB/s: 3 us of launch, 11,447 units for 4,864 warps, so a third turn of
// loads for a third of the warps, and no unit's loads before the last one's sum; the last CTA's sum).
#include <type_traits>

#include "ea_lm.cuh"

namespace ea {

constexpr int kNormThreads = 256;
constexpr int kNormCtasPerSm = 4;
constexpr int kNormWarps = kNormThreads / 32;
constexpr int kNormBytes = 4096;  // of a warp's unit of work: eight 16-byte loads per lane

struct NormArgs {
    int64_t units;           // of this launch
    int n_tensors;           // of this launch
    const int64_t *first;    // n_tensors + 1: each tensor's first unit within the launch
    const int64_t *sizes;
    double *partials;        // one per CTA, of this launch
    const double *all;       // of all launches, n_all of them
    int n_all;
    unsigned *ticket;
    int last;                // whether this launch is the last one
    float grad_scale, max_norm;
    float *out;
};

// The elements of 16 bytes as binary32.
__device__ __forceinline__ void unpack(const uint4 &v, float (&x)[4], const float *)
{
    x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
}
template <class G>
__device__ __forceinline__ void unpack(const uint4 &v, float (&x)[8], const G *)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (std::is_same<G, bf16>::value) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            x[2 * i] = f.x, x[2 * i + 1] = f.y;
        }
    }
}

// Sum of the squares of `count` elements from g on in binary64: any magnitude.
template <class G>
__device__ __noinline__ double wide_squares(const G *g, int count)
{
    double sum = 0.0;
    for (int i = 0; i < count; ++i) {
        const double x = to_f32(g[i]);
        sum += x * x;
    }
    return sum;
}

// The CTA's sum, in a fixed order, valid in thread 0.  One barrier before `red` may be reused.
__device__ __forceinline__ double norm_block_sum(double v, double *red)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    if (threadIdx.x == 0)
#pragma unroll
        for (int w = 0; w < kNormWarps; ++w) v += red[w];
    return v;
}

// A read-only pass: a warp takes units of kNormBytes of one tensor, its loads 16 bytes wide and all in flight at
// once (a tensor that starts off a 16-byte boundary gives its first elements to its first unit).  A lane's squares
// are formed and added in binary32, a few dozen of them, where their sum shows that none overflowed and that any that
// underflowed do not count; otherwise, and between units, in binary64.  Each CTA leaves one partial sum, and the
// last one to finish adds those in order.
template <class G>
__global__ void __launch_bounds__(kNormThreads, kNormCtasPerSm) norm_kernel(const NormArgs a, const __grid_constant__ GradList list)
{
    constexpr int kVec = 16 / sizeof(G), kPacks = kNormBytes / 512, kNormUnit = kNormBytes / sizeof(G);
    __shared__ double red[kNormWarps];
    __shared__ bool last;
    const int lane = threadIdx.x & 31;
    const int64_t warps = static_cast<int64_t>(gridDim.x) * kNormWarps;
    double sum = 0.0;
    int t = 0;
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * kNormWarps + (threadIdx.x >> 5); u < a.units; u += warps) {
        t = tensor_of(a.first, a.n_tensors, u, t);
        const G *g = static_cast<const G *>(list.g[t]);
        const int64_t size = a.sizes[t], unit = u - a.first[t];
        const int64_t off = (reinterpret_cast<uintptr_t>(g) & 15) / sizeof(G);  // elements after the boundary before g
        const int64_t begin = unit == 0 ? 0 : unit * kNormUnit - off;
        const int64_t end = u + 1 == a.first[t + 1] ? size : (unit + 1) * kNormUnit - off;
        const int64_t body = unit == 0 ? min(size, off ? kVec - off : 0) : begin;  // the first whole pack
        const int packs = static_cast<int>(min((end - body) / kVec, static_cast<int64_t>(32 * kPacks)));
        const uint4 *pack = reinterpret_cast<const uint4 *>(g + body) + lane;
        uint4 v[kPacks];
        if (packs == 32 * kPacks) {
#pragma unroll
            for (int k = 0; k < kPacks; ++k) v[k] = pack[32 * k];
        } else {
#pragma unroll
            for (int k = 0; k < kPacks; ++k) v[k] = 32 * k + lane < packs ? pack[32 * k] : make_uint4(0, 0, 0, 0);
        }
        float part = 0.0f;
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            float x[kVec], s = 0.0f;
            unpack(v[k], x, g);
#pragma unroll
            for (int i = 0; i < kVec; ++i) s = __fmaf_rn(x[i], x[i], s);
            part = __fadd_rn(part, s);
        }
        if (part >= 0x1p-80f && part < __int_as_float(0x7f800000)) {
            sum += part;
        } else {
            uint32_t any = 0;  // zeros are common, whole units of them
#pragma unroll
            for (int k = 0; k < kPacks; ++k) any |= v[k].x | v[k].y | v[k].z | v[k].w;
            if (any)
                for (int k = 0; 32 * k + lane < packs; ++k) sum += wide_squares(g + body + (32 * k + lane) * kVec, kVec);
        }
        // what is left on either side: fewer than kVec elements before, fewer than 2 kVec after (in the last unit)
        if (begin < body || body + packs * kVec < end) {
            const int64_t tail = body + packs * kVec, edge = lane < kVec ? begin + lane : tail + lane - kVec;
            if (lane < kVec ? edge < body : edge < end) sum += wide_squares(g + edge, 1);
        }
    }
    const double total = norm_block_sum(sum, red);
    if (threadIdx.x == 0) {
        a.partials[blockIdx.x] = total;
        __threadfence();
        last = a.last && atomicAdd(a.ticket, 1u) == gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    double v = 0.0;
    for (int i = threadIdx.x; i < a.n_all; i += kNormThreads) v += __ldcg(a.all + i);
    v = norm_block_sum(v, red);
    if (threadIdx.x == 0) {
        *a.ticket = 0;
        const double wide = fabs(static_cast<double>(a.grad_scale)) * sqrt(v);
        const float norm = static_cast<float>(wide);
        float factor = a.grad_scale;
        if (!isfinite(norm)) factor = __int_as_float(0x7fc00000);
        else if (norm > a.max_norm) factor = static_cast<float>(a.grad_scale * (a.max_norm / wide));
        a.out[0] = norm;
        a.out[1] = factor;
    }
}

}  // namespace ea

using namespace ea;

struct ea_norm {
    DeviceOf dev;
    cudaStream_t stream = nullptr;
    int32_t type = 0;
    std::vector<int64_t> sizes;
    struct Launch {
        int first_tensor, n_tensors, grid;
        int64_t units, first_at;  // first_at: of its unit offsets in the table
    };
    std::vector<Launch> launches;
    std::vector<int64_t> table;  // every launch's unit offsets (kept until the upload is done)
    int64_t *d_first = nullptr, *d_sizes = nullptr;
    double *d_partials = nullptr;
    unsigned *d_ticket = nullptr;
    int n_partials = 0;
};

namespace {

int validate(const ea_grad_norm_config *cfg)
{
    if (!cfg) return lm_fail(EA_E_INVAL, "config is NULL");
    if (cfg->n_tensors < 1 || cfg->n_tensors > (1 << 20)) return lm_fail(EA_E_INVAL, "n_tensors must be in [1, 2^20]");
    if (!cfg->sizes) return lm_fail(EA_E_INVAL, "sizes is NULL");
    if (!is_float_type(cfg->grad_type)) return lm_fail(EA_E_INVAL, "unknown gradient type %d", cfg->grad_type);
    for (int32_t i = 0; i < cfg->n_tensors; ++i)
        if (cfg->sizes[i] < 0 || cfg->sizes[i] > (int64_t{1} << 40))
            return lm_fail(EA_E_INVAL, "the size of tensor %d is out of [0, 2^40]", i);
    return EA_OK;
}

// Bytes of the pieces of the workspace, each a multiple of 256.
struct NormLayout {
    size_t first, sizes, partials, ticket;
    size_t total() const { return first + sizes + partials + ticket; }
};

NormLayout norm_layout(const ea_grad_norm_config &cfg, int sms)
{
    const size_t n = cfg.n_tensors, launches = (n + kGradBatch - 1) / kGradBatch;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    return {up((n + launches) * 8), up(n * 8), up(launches * sms * kNormCtasPerSm * 8), up(4)};
}

}  // namespace

extern "C" {

int ea_grad_norm_workspace_bytes(const ea_grad_norm_config *cfg, size_t *bytes)
{
    if (!bytes) return lm_fail(EA_E_INVAL, "bytes is NULL");
    const int r = validate(cfg);
    if (r != EA_OK) return r;
    *bytes = norm_layout(*cfg, kMaxSms).total();
    return EA_OK;
}

int ea_grad_norm_init(const ea_grad_norm_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_norm **out)
{
    if (!out) return lm_fail(EA_E_INVAL, "out is NULL");
    *out = nullptr;
    int r = validate(cfg);
    if (r != EA_OK) return r;
    const NormLayout L = norm_layout(*cfg, kMaxSms);
    if ((r = check_workspace(workspace, workspace_bytes, L.total())) != EA_OK) return r;
    DeviceOf dev;
    if ((r = dev.query()) != EA_OK) return r;
    ea_norm *h = new (std::nothrow) ea_norm;
    if (!h) return lm_fail(EA_E_INVAL, "out of host memory");
    h->dev = dev;
    try {
        h->stream = static_cast<cudaStream_t>(stream);
        h->type = cfg->grad_type;
        h->sizes.assign(cfg->sizes, cfg->sizes + cfg->n_tensors);
        for (int i = 0; i < cfg->n_tensors; i += kGradBatch) {
            ea_norm::Launch l{i, std::min(kGradBatch, cfg->n_tensors - i), 0, 0, static_cast<int64_t>(h->table.size())};
            const int64_t unit = kNormBytes / static_cast<int64_t>(type_bytes(cfg->grad_type));
            for (int k = 0; k < l.n_tensors; ++k) {
                h->table.push_back(l.units);
                l.units += (h->sizes[i + k] + unit - 1) / unit;
            }
            h->table.push_back(l.units);
            const int64_t ctas = (l.units + kNormThreads / 32 - 1) / (kNormThreads / 32);
            l.grid = static_cast<int>(std::clamp<int64_t>(ctas, 1, std::min(h->dev.sms, kMaxSms) * kNormCtasPerSm));
            h->n_partials += l.grid;
            h->launches.push_back(l);
        }
    } catch (const std::bad_alloc &) {
        r = lm_fail(EA_E_INVAL, "out of host memory");
    }
    if (r == EA_OK) {
        char *p = static_cast<char *>(workspace);
        h->d_first = reinterpret_cast<int64_t *>(p);
        h->d_sizes = reinterpret_cast<int64_t *>(p += L.first);
        h->d_partials = reinterpret_cast<double *>(p += L.sizes);
        h->d_ticket = reinterpret_cast<unsigned *>(p += L.partials);
        r = lm_cuda(cudaMemsetAsync(h->d_ticket, 0, 4, h->stream), "ticket clear");
    }
    if (r == EA_OK)
        r = lm_cuda(cudaMemcpyAsync(h->d_first, h->table.data(), h->table.size() * 8, cudaMemcpyHostToDevice, h->stream), "table upload");
    if (r == EA_OK)
        r = lm_cuda(cudaMemcpyAsync(h->d_sizes, h->sizes.data(), h->sizes.size() * 8, cudaMemcpyHostToDevice, h->stream), "table upload");
    if (r != EA_OK) {
        delete h;
        return r;
    }
    *out = h;
    return EA_OK;
}

int ea_grad_norm(ea_norm *h, const void *const *grads, float grad_scale, float max_norm, float *out)
{
    if (!h) return lm_fail(EA_E_INVAL, "handle is NULL");
    if (!grads) return lm_fail(EA_E_INVAL, "grads is NULL");
    if (!std::isfinite(grad_scale) || grad_scale == 0.0f) return lm_fail(EA_E_INVAL, "grad_scale must be finite and not 0");
    if (!(max_norm >= 0.0f)) return lm_fail(EA_E_INVAL, "max_norm must be >= 0");
    int r = check_address(out, EA_T_F32, "out");
    for (size_t i = 0; r == EA_OK && i < h->sizes.size(); ++i)
        if (h->sizes[i]) r = check_address(grads[i], h->type, "a gradient");
    if (r == EA_OK) r = h->dev.check();
    if (r != EA_OK) return r;
    int at = 0;
    for (size_t k = 0; k < h->launches.size(); ++k) {
        const ea_norm::Launch &l = h->launches[k];
        GradList list{};
        std::copy(grads + l.first_tensor, grads + l.first_tensor + l.n_tensors, list.g);
        const NormArgs a{l.units, l.n_tensors, h->d_first + l.first_at, h->d_sizes + l.first_tensor, h->d_partials + at,
                         h->d_partials, h->n_partials, h->d_ticket, k + 1 == h->launches.size(), grad_scale, max_norm, out};
        switch (h->type) {
        case EA_T_F32: norm_kernel<float><<<l.grid, kNormThreads, 0, h->stream>>>(a, list); break;
        case EA_T_BF16: norm_kernel<bf16><<<l.grid, kNormThreads, 0, h->stream>>>(a, list); break;
        default: norm_kernel<f16><<<l.grid, kNormThreads, 0, h->stream>>>(a, list);
        }
        if ((r = lm_cuda(cudaGetLastError(), "launch")) != EA_OK) return r;
        at += l.grid;
    }
    return EA_OK;
}

int ea_grad_norm_destroy(ea_norm *h)
{
    delete h;
    return EA_OK;
}

}  // extern "C"
