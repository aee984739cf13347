// ea_embed.cu -- the lookup of tokens in an embedding table (ea_embed_lookup) and the gradient of the table
// (ea_embed_grad).
#include "ea_lm.cuh"

namespace ea {

constexpr uint32_t kStatusToken = 4u;  // a token outside the table
constexpr int kEmbedThreads = 256;

struct EmbedArgs {
    int64_t n, inner;            // tokens; tokens per row of the batch
    int64_t token_outer, token_inner, row_outer, row_inner, table_stride;
    int64_t vocab, dim, padding;
    float scale;
    int token64;
    const void *tokens;
    uint32_t *status;
};

__device__ __forceinline__ int64_t token_at(const EmbedArgs &a, int64_t t)
{
    const int64_t i = t / a.inner, at = i * a.token_outer + (t - i * a.inner) * a.token_inner;
    return a.token64 ? static_cast<const int64_t *>(a.tokens)[at] : static_cast<const int32_t *>(a.tokens)[at];
}

__device__ __forceinline__ int64_t row_at(const EmbedArgs &a, int64_t t)
{
    const int64_t i = t / a.inner;
    return i * a.row_outer + (t - i * a.inner) * a.row_inner;
}

// One CTA per token.
template <class W, class Y>
__global__ void __launch_bounds__(kEmbedThreads) lookup_kernel(const EmbedArgs a, const W *w, Y *y)
{
    for (int64_t t = blockIdx.x; t < a.n; t += gridDim.x) {
        const int64_t v = token_at(a, t);
        Y *row = y + row_at(a, t);
        const bool inside = v >= 0 && v < a.vocab;
        if (!inside && threadIdx.x == 0) atomicOr(a.status, kStatusToken);
        for (int64_t j = threadIdx.x; j < a.dim; j += kEmbedThreads)
            row[j] = from_f32<Y>(inside ? __fmul_rn(to_f32(w[v * a.table_stride + j]), a.scale) : 0.0f);
    }
}

// One CTA per row of the table: it goes through all tokens.
template <class Y, class W>
__global__ void __launch_bounds__(kEmbedThreads) grad_kernel(const EmbedArgs a, const Y *dy, W *dw, int accumulate)
{
    for (int64_t v = blockIdx.x; v < a.vocab; v += gridDim.x) {
        for (int64_t j0 = 0; j0 < a.dim; j0 += kEmbedThreads) {
            const int64_t j = j0 + threadIdx.x;
            float sum = 0.0f;
            bool any = false;
            if (v != a.padding)
                for (int64_t t = 0; t < a.n; ++t)
                    if (token_at(a, t) == v) {
                        any = true;
                        if (j < a.dim) sum = __fadd_rn(sum, to_f32(dy[row_at(a, t) + j]));
                    }
            if (j < a.dim && (any || !accumulate)) {
                W &out = dw[v * a.table_stride + j];
                sum = __fmul_rn(sum, a.scale);
                out = from_f32<W>(accumulate ? __fadd_rn(to_f32(out), sum) : sum);
            }
        }
    }
}

__global__ void __launch_bounds__(kEmbedThreads) check_tokens_kernel(const EmbedArgs a)
{
    for (int64_t t = blockIdx.x * static_cast<int64_t>(kEmbedThreads) + threadIdx.x; t < a.n;
         t += static_cast<int64_t>(gridDim.x) * kEmbedThreads) {
        const int64_t v = token_at(a, t);
        if (v < 0 || v >= a.vocab) atomicOr(a.status, kStatusToken);
    }
}

}  // namespace ea

using namespace ea;

struct ea_embed {
    DeviceOf dev;
    cudaStream_t stream = nullptr;
    ea_embed_config cfg{};
    uint32_t *status = nullptr;
};

namespace {

int validate(const ea_embed_config *cfg)
{
    if (!cfg) return lm_fail(EA_E_INVAL, "config is NULL");
    if (cfg->vocab < 1 || cfg->vocab > 0x7ffffffeLL) return lm_fail(EA_E_INVAL, "vocab must be in [1, 2^31 - 2]");
    if (cfg->dim < 1 || cfg->dim > (1 << 24)) return lm_fail(EA_E_INVAL, "dim must be in [1, 2^24]");
    if (cfg->max_tokens < 0 || cfg->max_tokens > (1 << 30)) return lm_fail(EA_E_INVAL, "max_tokens must be in [0, 2^30]");
    if (cfg->padding < -1 || cfg->padding >= cfg->vocab) return lm_fail(EA_E_INVAL, "padding must be a token or -1");
    if (!std::isfinite(cfg->scale)) return lm_fail(EA_E_INVAL, "scale must be finite");
    return EA_OK;
}

size_t embed_bytes(const ea_embed_config &) { return 256; }

// Checks a call and fills in the kernels' arguments.
int embed_args(const ea_embed *h, const ea_embed_call *c, const void *tokens, const void *rows, const void *table,
               EmbedArgs &a)
{
    if (!h) return lm_fail(EA_E_INVAL, "handle is NULL");
    if (!c) return lm_fail(EA_E_INVAL, "call is NULL");
    if (c->outer < 0 || c->inner < 0 || (c->inner && c->outer > h->cfg.max_tokens / c->inner))
        return lm_fail(EA_E_INVAL, "%lld x %lld tokens: the handle takes up to %lld", static_cast<long long>(c->outer),
                       static_cast<long long>(c->inner), static_cast<long long>(h->cfg.max_tokens));
    if (c->token_type != EA_T_I32 && c->token_type != EA_T_I64) return lm_fail(EA_E_INVAL, "tokens are 32- or 64-bit integers");
    if (!is_float_type(c->row_type)) return lm_fail(EA_E_INVAL, "unknown row type %d", c->row_type);
    if (!is_float_type(c->table_type)) return lm_fail(EA_E_INVAL, "unknown table type %d", c->table_type);
    if (c->table_stride < h->cfg.dim) return lm_fail(EA_E_INVAL, "the table's rows overlap");
    int r = check_address(table, c->table_type, "the table");
    if (c->outer * c->inner) {
        if (r == EA_OK) r = check_address(tokens, c->token_type, "tokens");
        if (r == EA_OK) r = check_address(rows, c->row_type, "the rows");
    }
    if (r == EA_OK) r = h->dev.check();
    if (r != EA_OK) return r;
    a = EmbedArgs{c->outer * c->inner, c->inner, c->token_outer, c->token_inner, c->row_outer, c->row_inner, c->table_stride,
                  h->cfg.vocab, h->cfg.dim, h->cfg.padding, h->cfg.scale, c->token_type == EA_T_I64, tokens, h->status};
    return EA_OK;
}

// f(a pointer of the element type) for the type at hand.
template <class F>
void with_type(int32_t type, F f)
{
    switch (type) {
    case EA_T_F32: f(static_cast<float *>(nullptr)); break;
    case EA_T_BF16: f(static_cast<bf16 *>(nullptr)); break;
    default: f(static_cast<f16 *>(nullptr));
    }
}

}  // namespace

extern "C" {

int ea_embed_workspace_bytes(const ea_embed_config *cfg, size_t *bytes)
{
    if (!bytes) return lm_fail(EA_E_INVAL, "bytes is NULL");
    const int r = validate(cfg);
    if (r != EA_OK) return r;
    *bytes = embed_bytes(*cfg);
    return EA_OK;
}

int ea_embed_init(const ea_embed_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_embed **out)
{
    if (!out) return lm_fail(EA_E_INVAL, "out is NULL");
    *out = nullptr;
    int r = validate(cfg);
    if (r != EA_OK) return r;
    if ((r = check_workspace(workspace, workspace_bytes, embed_bytes(*cfg))) != EA_OK) return r;
    ea_embed *h = new (std::nothrow) ea_embed;
    if (!h) return lm_fail(EA_E_INVAL, "out of host memory");
    h->cfg = *cfg;
    h->stream = static_cast<cudaStream_t>(stream);
    h->status = static_cast<uint32_t *>(workspace);
    r = h->dev.query();
    if (r == EA_OK) r = lm_cuda(cudaMemsetAsync(h->status, 0, 4, h->stream), "status clear");
    if (r != EA_OK) {
        delete h;
        return r;
    }
    *out = h;
    return EA_OK;
}

int ea_embed_lookup(ea_embed *h, const ea_embed_call *c, const void *tokens, const void *w, void *y)
{
    EmbedArgs a;
    const int r = embed_args(h, c, tokens, y, w, a);
    if (r != EA_OK || a.n == 0) return r;
    with_type(c->table_type, [&](auto *wt) {
        with_type(c->row_type, [&](auto *yt) {
            lookup_kernel<<<static_cast<unsigned>(std::min<int64_t>(a.n, 1 << 20)), kEmbedThreads, 0, h->stream>>>(
                a, static_cast<decltype(wt)>(const_cast<void *>(w)), static_cast<decltype(yt)>(y));
        });
    });
    return lm_cuda(cudaGetLastError(), "launch");
}

int ea_embed_grad(ea_embed *h, const ea_embed_call *c, const void *tokens, const void *dy, void *dw, int32_t accumulate)
{
    if (accumulate != 0 && accumulate != 1) return lm_fail(EA_E_INVAL, "accumulate is 0 or 1");
    EmbedArgs a;
    const int r = embed_args(h, c, tokens, dy, dw, a);
    if (r != EA_OK) return r;
    with_type(c->row_type, [&](auto *yt) {
        with_type(c->table_type, [&](auto *wt) {
            grad_kernel<<<static_cast<unsigned>(std::min<int64_t>(a.vocab, 1 << 20)), kEmbedThreads, 0, h->stream>>>(
                a, static_cast<decltype(yt)>(const_cast<void *>(dy)), static_cast<decltype(wt)>(dw), accumulate);
        });
    });
    if (a.n) check_tokens_kernel<<<static_cast<unsigned>(std::min<int64_t>((a.n + 255) / 256, 1024)), kEmbedThreads, 0, h->stream>>>(a);
    return lm_cuda(cudaGetLastError(), "launch");
}

int ea_embed_sync_status(ea_embed *h)
{
    if (!h) return lm_fail(EA_E_INVAL, "handle is NULL");
    uint32_t st = 0;
    int r = lm_cuda(cudaMemcpyAsync(&st, h->status, 4, cudaMemcpyDeviceToHost, h->stream), "status read");
    if (r == EA_OK) r = lm_cuda(cudaMemsetAsync(h->status, 0, 4, h->stream), "status clear");
    if (r == EA_OK) r = lm_cuda(cudaStreamSynchronize(h->stream), "stream synchronize");
    if (r != EA_OK) return r;
    if (st & kStatusToken) return lm_fail(EA_E_DEVICE_CHECK, "a token lay outside [0, %lld)", static_cast<long long>(h->cfg.vocab));
    return EA_OK;
}

int ea_embed_destroy(ea_embed *h)
{
    delete h;
    return EA_OK;
}

}  // extern "C"
