// ea_scan.cu -- ea_scan_forward and ea_scan_backward.
#include "ea_block.cuh"

namespace ea {

constexpr uint32_t kStatusLength = 8u;  // a length outside [0, length]
constexpr int kScanThreads = 128;

struct ScanArgs {
    int64_t batch, length, dim, columns;  // columns = batch * dim
    const float *initial;
    const void *lengths;
    int length64;
    uint32_t *status;
};

// A sequence's length within [0, length].
__device__ __forceinline__ int64_t scan_length(const ScanArgs &a, int64_t i)
{
    if (!a.lengths) return a.length;
    const int64_t n = a.length64 ? static_cast<const int64_t *>(a.lengths)[i] : static_cast<const int32_t *>(a.lengths)[i];
    if (n < 0 || n > a.length) atomicOr(a.status, kStatusLength);
    return n < 0 ? 0 : n > a.length ? a.length : n;
}

// f = 1 / (1 + e^-z) and 1 - f = e^-z / (1 + e^-z), each with a small relative error at either end.
__device__ __forceinline__ void gate(float z, float &f, float &shut)
{
    const float e = __expf(-fabsf(z)), big = __fdividef(1.0f, __fadd_rn(1.0f, e)), small = __fmul_rn(e, big);
    f = z >= 0.0f ? big : small;
    shut = z >= 0.0f ? small : big;
}

// One thread takes a column of a sequence from its first row to its last.
template <class T>
__global__ void __launch_bounds__(kScanThreads) scan_forward_kernel(const ScanArgs a, const T *z, int64_t z_batch, int64_t z_row, const T *v, int64_t v_batch,
                                                                    int64_t v_row, T *h, int64_t h_batch, int64_t h_row, float *final)
{
    const int64_t k = static_cast<int64_t>(blockIdx.x) * kScanThreads + threadIdx.x;
    if (k >= a.columns) return;
    const int64_t i = k / a.dim, c = k - i * a.dim, n = scan_length(a, i);
    z += i * z_batch + c, v += i * v_batch + c, h += i * h_batch + c;
    float state = a.initial ? a.initial[k] : 0.0f;
    int64_t t = 0;
    for (; t < n; ++t) {
        float f, shut;
        gate(to_f32(z[t * z_row]), f, shut);
        state = __fmaf_rn(f, state, __fmul_rn(shut, to_f32(v[t * v_row])));
        h[t * h_row] = from_f32<T>(state);
    }
    for (; t < a.length; ++t) h[t * h_row] = from_f32<T>(0.0f);
    if (final) final[k] = state;
}

template <class T>
__global__ void __launch_bounds__(kScanThreads) scan_backward_kernel(const ScanArgs a, const ea_scan_call s, const T *dh, const T *z, const T *v, const T *h,
                                                                     const float *d_final, T *dz, T *dv, float *d_initial)
{
    const int64_t k = static_cast<int64_t>(blockIdx.x) * kScanThreads + threadIdx.x;
    if (k >= a.columns) return;
    const int64_t i = k / a.dim, c = k - i * a.dim, n = scan_length(a, i);
    dh += i * s.dh_batch + c, z += i * s.z_batch + c, v += i * s.v_batch + c, h += i * s.h_batch + c;
    dz += i * s.dz_batch + c, dv += i * s.dv_batch + c;
    int64_t t = a.length - 1;
    for (; t >= n; --t) dz[t * s.dz_row] = dv[t * s.dv_row] = from_f32<T>(0.0f);
    float later = d_final ? d_final[k] : 0.0f;  // f_{t+1} g_{t+1}
    for (; t >= 0; --t) {
        float f, shut;
        gate(to_f32(z[t * s.z_row]), f, shut);
        const float g = __fadd_rn(to_f32(dh[t * s.dh_row]), later);
        const float before = t ? to_f32(h[(t - 1) * s.h_row]) : a.initial ? a.initial[k] : 0.0f;
        const float dvt = __fmul_rn(shut, g);
        later = __fmul_rn(f, g);
        const float dzt = __fmul_rn(__fmul_rn(f, dvt), __fsub_rn(before, to_f32(v[t * s.v_row])));
        dz[t * s.dz_row] = from_f32<T>(dzt);
        dv[t * s.dv_row] = from_f32<T>(dvt);
    }
    if (d_initial) d_initial[k] = later;
}

}  // namespace ea

using namespace ea;

struct ea_scan {
    ea_scan_config cfg{};
    DeviceOf dev;
    cudaStream_t stream = nullptr;
    uint32_t *status = nullptr;
};

namespace {

constexpr size_t kScanBytes = 256;

int validate(const ea_scan_config *cfg)
{
    if (!cfg) return lm_fail(EA_E_INVAL, "config is NULL");
    if (cfg->dim < 1 || cfg->dim > (int64_t{1} << 20)) return lm_fail(EA_E_INVAL, "dim must be in [1, 2^20]");
    return EA_OK;
}

int check_call(const ea_scan *s, const ea_scan_call *c, const float *initial, const void *lengths, ScanArgs &a)
{
    if (!s) return lm_fail(EA_E_INVAL, "handle is NULL");
    if (!c) return lm_fail(EA_E_INVAL, "call is NULL");
    if (c->batch < 0 || c->batch > (int64_t{1} << 24) || c->length < 0 || c->length > kMaxRows || c->batch * s->cfg.dim >= (int64_t{1} << 31))
        return lm_fail(EA_E_INVAL, "%lld sequences of %lld rows of %lld: out of range", static_cast<long long>(c->batch), static_cast<long long>(c->length),
                       static_cast<long long>(s->cfg.dim));
    if (!is_float_type(c->type)) return lm_fail(EA_E_INVAL, "unknown type %d", c->type);
    if (lengths && c->length_type != EA_T_I32 && c->length_type != EA_T_I64) return lm_fail(EA_E_INVAL, "lengths are 32- or 64-bit integers");
    int r = EA_OK;
    if (initial) r = check_address(initial, EA_T_F32, "initial");
    if (r == EA_OK && lengths) r = check_address(lengths, c->length_type, "lengths");
    if (r == EA_OK) r = s->dev.check();
    if (r != EA_OK) return r;
    a = ScanArgs{c->batch, c->length, s->cfg.dim, c->batch * s->cfg.dim, initial, lengths, c->length_type == EA_T_I64, s->status};
    return EA_OK;
}

}  // namespace

extern "C" {

int ea_scan_workspace_bytes(const ea_scan_config *cfg, size_t *bytes)
{
    if (!bytes) return lm_fail(EA_E_INVAL, "bytes is NULL");
    const int r = validate(cfg);
    if (r != EA_OK) return r;
    *bytes = kScanBytes;
    return EA_OK;
}

int ea_scan_init(const ea_scan_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_scan **out)
{
    if (!out) return lm_fail(EA_E_INVAL, "out is NULL");
    *out = nullptr;
    int r = validate(cfg);
    if (r != EA_OK) return r;
    if ((r = check_workspace(workspace, workspace_bytes, kScanBytes)) != EA_OK) return r;
    DeviceOf dev;
    if ((r = dev.query()) != EA_OK) return r;
    if ((r = lm_cuda(cudaMemsetAsync(workspace, 0, 4, static_cast<cudaStream_t>(stream)), "status clear")) != EA_OK) return r;
    ea_scan *s = new (std::nothrow) ea_scan;
    if (!s) return lm_fail(EA_E_INVAL, "out of host memory");
    s->cfg = *cfg;
    s->dev = dev;
    s->stream = static_cast<cudaStream_t>(stream);
    s->status = static_cast<uint32_t *>(workspace);
    *out = s;
    return EA_OK;
}

int ea_scan_forward(ea_scan *s, const ea_scan_call *c, const void *z, const void *v, const float *initial, const void *lengths, void *h, float *final)
{
    ScanArgs a;
    int r = check_call(s, c, initial, lengths, a);
    if (r != EA_OK) return r;
    if (final) r = check_address(final, EA_T_F32, "final");
    if (a.columns && a.length) {
        if (r == EA_OK) r = check_address(z, c->type, "z");
        if (r == EA_OK) r = check_address(v, c->type, "v");
        if (r == EA_OK) r = check_address(h, c->type, "h");
        if (r == EA_OK) r = check_rows_apart(a.batch, a.length, c->h_batch, c->h_row, a.dim, "h");
    }
    if (r != EA_OK || !a.columns || (!a.length && !final)) return r;
    with_float(c->type, [&](auto *t) {
        using T = std::remove_reference_t<decltype(*t)>;
        scan_forward_kernel<T><<<static_cast<unsigned>(over<int64_t>(a.columns, kScanThreads)), kScanThreads, 0, s->stream>>>(
            a, static_cast<const T *>(z), c->z_batch, c->z_row, static_cast<const T *>(v), c->v_batch, c->v_row, static_cast<T *>(h), c->h_batch, c->h_row, final);
    });
    return lm_cuda(cudaGetLastError(), "launch");
}

int ea_scan_backward(ea_scan *s, const ea_scan_call *c, const void *dh, const void *z, const void *v, const void *h, const float *initial,
                     const void *lengths, const float *d_final, void *dz, void *dv, float *d_initial)
{
    ScanArgs a;
    int r = check_call(s, c, initial, lengths, a);
    if (r != EA_OK) return r;
    if (d_final) r = check_address(d_final, EA_T_F32, "d_final");
    if (r == EA_OK && d_initial) r = check_address(d_initial, EA_T_F32, "d_initial");
    if (a.columns && a.length) {
        const std::pair<const void *, const char *> all[] = {{dh, "dh"}, {z, "z"}, {v, "v"}, {h, "h"}, {dz, "dz"}, {dv, "dv"}};
        for (const auto &p : all)
            if (r == EA_OK) r = check_address(p.first, c->type, p.second);
        if (r == EA_OK) r = check_rows_apart(a.batch, a.length, c->dz_batch, c->dz_row, a.dim, "dz");
        if (r == EA_OK) r = check_rows_apart(a.batch, a.length, c->dv_batch, c->dv_row, a.dim, "dv");
        if (r == EA_OK && (dz == h || dv == h || dz == dv)) r = lm_fail(EA_E_INVAL, "dz and dv may be neither h nor one another");
    }
    if (r != EA_OK || !a.columns || (!a.length && !d_initial)) return r;
    with_float(c->type, [&](auto *t) {
        using T = std::remove_reference_t<decltype(*t)>;
        scan_backward_kernel<T><<<static_cast<unsigned>(over<int64_t>(a.columns, kScanThreads)), kScanThreads, 0, s->stream>>>(
            a, *c, static_cast<const T *>(dh), static_cast<const T *>(z), static_cast<const T *>(v), static_cast<const T *>(h), d_final,
            static_cast<T *>(dz), static_cast<T *>(dv), d_initial);
    });
    return lm_cuda(cudaGetLastError(), "launch");
}

int ea_scan_sync_status(ea_scan *s)
{
    if (!s) return lm_fail(EA_E_INVAL, "handle is NULL");
    uint32_t st = 0;
    int r = lm_cuda(cudaMemcpyAsync(&st, s->status, 4, cudaMemcpyDeviceToHost, s->stream), "status read");
    if (r == EA_OK) r = lm_cuda(cudaMemsetAsync(s->status, 0, 4, s->stream), "status clear");
    if (r == EA_OK) r = lm_cuda(cudaStreamSynchronize(s->stream), "stream synchronize");
    if (r != EA_OK) return r;
    if (st & kStatusLength) return lm_fail(EA_E_DEVICE_CHECK, "a sequence's length lay outside its rows");
    return EA_OK;
}

int ea_scan_destroy(ea_scan *s)
{
    delete s;
    return EA_OK;
}

}  // extern "C"
