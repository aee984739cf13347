// ea_adamw.cu -- ea_adamw_step: one AdamW step (Loshchilov and Hutter; Adam's bias correction folded into the
// step size and epsilon as in the last remark of Kingma and Ba's Section 2) over a list of tensors, with
// moments in binary32 or in 8 bits.
#include <cuda_fp8.h>

#include "ea_device.cuh"
#include "ea_lm.cuh"

namespace ea {

constexpr int kAdamThreads = 256;
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
    uint64_t seed;
    const float *clip;
};

__device__ __forceinline__ uint32_t e4m3_code(float x, float inv, uint32_t r16, bool keep_nonzero)
{
    const uint32_t bits = __float_as_uint(x) & 0x7fffffffu;
    if (bits >= 0x7f800000u) return 0x7fu;  // not finite: NaN
    const float y = __fmul_rn(__uint_as_float(bits), inv);
    uint32_t code;
    if (y >= 0x1p-6f) code = ((__float_as_uint(y) + (r16 << 4)) >> 20) - ((127u - 7u) << 3);
    else code = static_cast<uint32_t>(floorf(__fadd_rn(__fmul_rn(y, 512.0f), __fmul_rn(static_cast<float>(r16), 0x1p-16f))));
    if (keep_nonzero && bits != 0 && code == 0) code = 1;
    return code | (__float_as_uint(x) >> 31 << 7);
}

__device__ __forceinline__ float e4m3_value(uint32_t code)
{
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(code), __NV_E4M3)));
}

// The exponent k of the smallest power of two >= 2^-126 with amax / 2^k <= 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(uint32_t amax_bits)
{
    return max(static_cast<int>((amax_bits + 0x1fffffu) >> 23) - 127 - 8, -126);
}

__device__ __forceinline__ uint32_t finite_magnitude(float x)
{
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

template <class P, class G, class C, int BITS>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const AdamArgs a, const __grid_constant__ GradList list)
{
    const int lane = threadIdx.x & 31;
    const float factor = a.clip ? a.clip[1] : 1.0f;
    const AdamState st = *a.state;
    if (!isnan(factor)) {
        const int64_t warps = static_cast<int64_t>(gridDim.x) * (kAdamThreads / 32);
        for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kAdamThreads / 32) + (threadIdx.x >> 5); u < a.units; u += warps) {
            int lo = 0, hi = a.n_tensors - 1;  // the last tensor whose first block is <= u
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (a.first[mid] <= u) lo = mid;
                else hi = mid - 1;
            }
            const ea_adamw_tensor &T = a.tensors[lo];
            const int64_t block = u - a.first[lo], base = block * kBlock;
            const int n = static_cast<int>(min(T.size - base, static_cast<int64_t>(kBlock)));
            const float lr = __fmul_rn(a.lr, T.lr_scale), step = __fmul_rn(lr, st.a), rate = __fmul_rn(lr, T.weight_decay);
            P *p = static_cast<P *>(T.param) + base;
            C *copy = T.copy ? static_cast<C *>(T.copy) + base : nullptr;
            const G *g = static_cast<const G *>(list.g[lo]) + base;
            float m[8], v[8], root[8];
            float ms = 1.0f, vs = 1.0f;
            if (BITS == 8) {
                ms = T.m_scale[block];
                vs = T.v_scale[block];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int j = (k >> 2) * 128 + lane * 4 + (k & 3);
                m[k] = v[k] = root[k] = 0.0f;
                if (j >= n) continue;
                const float gk = __fmul_rn(to_f32(g[j]), factor);
                if (BITS == 32) {
                    m[k] = static_cast<const float *>(T.m)[base + j];
                    v[k] = static_cast<const float *>(T.v)[base + j];
                } else {
                    m[k] = __fmul_rn(e4m3_value(static_cast<const uint8_t *>(T.m)[base + j]), ms);
                    const float r = __fmul_rn(e4m3_value(static_cast<const uint8_t *>(T.v)[base + j]), vs);
                    v[k] = __fmul_rn(r, r);
                }
                m[k] = __fadd_rn(__fmul_rn(m[k], a.beta1), __fmul_rn(gk, a.c1));
                v[k] = __fadd_rn(__fmul_rn(v[k], a.beta2), __fmul_rn(__fmul_rn(gk, gk), a.c2));
                root[k] = __fsqrt_rn(v[k]);
                const float pk = to_f32(p[j]);
                const float d = __fadd_rn(__fmul_rn(pk, rate), __fmul_rn(__fdiv_rn(m[k], __fadd_rn(root[k], st.e)), step));
                const float q = __fsub_rn(pk, d);
                p[j] = from_f32<P>(q);
                if (copy) copy[j] = from_f32<C>(q);
                if (BITS == 32) {
                    static_cast<float *>(T.m)[base + j] = m[k];
                    static_cast<float *>(T.v)[base + j] = v[k];
                }
            }
            if (BITS == 8) {
                uint32_t am = 0, av = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    am = max(am, finite_magnitude(m[k]));
                    av = max(av, finite_magnitude(root[k]));
                }
                const int km = scale_exponent(__reduce_max_sync(0xffffffffu, am));
                const int kv = scale_exponent(__reduce_max_sync(0xffffffffu, av));
                const float im = __uint_as_float(static_cast<uint32_t>(127 - km) << 23);
                const float iv = __uint_as_float(static_cast<uint32_t>(127 - kv) << 23);
                if (lane == 0) {
                    T.m_scale[block] = __uint_as_float(static_cast<uint32_t>(127 + km) << 23);
                    T.v_scale[block] = __uint_as_float(static_cast<uint32_t>(127 + kv) << 23);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int j0 = h * 128 + lane * 4;
                    if (j0 >= n) continue;
                    const uint64_t quad = static_cast<uint64_t>(base + j0) >> 2;
                    const uint4 w = philox4x32_10(make_uint4(static_cast<uint32_t>(quad), static_cast<uint32_t>(quad >> 32),
                                                             static_cast<uint32_t>(a.tensor0 + lo), static_cast<uint32_t>(st.t)),
                                                  make_uint2(static_cast<uint32_t>(a.seed), static_cast<uint32_t>(a.seed >> 32)));
                    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (j0 + i >= n) continue;
                        static_cast<uint8_t *>(T.m)[base + j0 + i] = static_cast<uint8_t>(e4m3_code(m[4 * h + i], im, word[i] & 0xffffu, false));
                        static_cast<uint8_t *>(T.v)[base + j0 + i] = static_cast<uint8_t>(e4m3_code(root[4 * h + i], iv, word[i] >> 16, true));
                    }
                }
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

constexpr int kAdamCtasPerSm = 4;

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
    if (!(cfg->eps > 0.0f) || !std::isfinite(cfg->eps)) return lm_fail(EA_E_INVAL, "eps must be > 0");
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
        a.seed = h->cfg.seed;
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
