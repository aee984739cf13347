// ea_scan.cu -- ea_scan_forward and ea_scan_backward.
//
// h_t = f_t h_{t-1} + u_t composes: two pieces (A, B) and (A', B') of a sequence, each standing for h -> A h + B, are together
// (A' A, A' B + B').  A cluster of CTAs takes the same columns of one sequence and walks along it, every CTA a chunk of rows at a
// step: threads compose their rows, warps and CTAs compose what those left, the cluster's CTAs exchange theirs, and every
// thread then runs through its rows again from the state that it starts with.  Each value is read once and written once.
// The gradient is the same recurrence from the last row to the first, c_t = f_t (dh_t + c_{t+1}).
#include "ea_async.cuh"
#include "ea_block.cuh"

namespace ea {

constexpr uint32_t kStatusLength = 8u;  // a length outside [0, length]
constexpr int kWalkThreads = 128;
constexpr int kTileThreads = 128, kTileWarps = kTileThreads / 32;
constexpr int kMaxCluster = 16;

// A tensor: element 0 of row t of sequence i at p + i * batch + t * row.
template <class T>
struct Seq {
    T *p;
    int64_t batch, row;
};

struct ScanArgs {
    int64_t batch, length, dim;
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

// V consecutive elements in one access.
template <class T, int V>
struct alignas(V * sizeof(T)) Vec {
    T x[V];
};

// ---------------------------------------------------------------------------------------------- short sequences
// A thread takes V columns of a sequence from its first row to its last, the loads of kAhead rows before their arithmetic.
constexpr int kAhead = 4;

template <class T, int V>
__global__ void __launch_bounds__(kWalkThreads) scan_walk_kernel(const ScanArgs a, const Seq<const T> zs, const Seq<const T> vs, const Seq<T> hs, float *final)
{
    const int64_t packs = a.dim / V, k = static_cast<int64_t>(blockIdx.x) * kWalkThreads + threadIdx.x;
    if (k >= a.batch * packs) return;
    const int64_t i = k / packs, c = (k - i * packs) * V, n = scan_length(a, i);
    const T *z = zs.p + i * zs.batch + c, *v = vs.p + i * vs.batch + c;
    T *h = hs.p + i * hs.batch + c;
    float state[V];
#pragma unroll
    for (int j = 0; j < V; ++j) state[j] = a.initial ? a.initial[i * a.dim + c + j] : 0.0f;
    for (int64_t t = 0; t < a.length; t += kAhead) {
        Vec<T, V> zv[kAhead], vv[kAhead], out;
#pragma unroll
        for (int r = 0; r < kAhead; ++r)
            if (t + r < n) {
                zv[r] = *reinterpret_cast<const Vec<T, V> *>(z + (t + r) * zs.row);
                vv[r] = *reinterpret_cast<const Vec<T, V> *>(v + (t + r) * vs.row);
            }
#pragma unroll
        for (int r = 0; r < kAhead; ++r) {
            if (t + r >= a.length) break;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float f, shut;
                if (t + r < n) {
                    gate(to_f32(zv[r].x[j]), f, shut);
                    state[j] = __fmaf_rn(f, state[j], __fmul_rn(shut, to_f32(vv[r].x[j])));
                }
                out.x[j] = from_f32<T>(t + r < n ? state[j] : 0.0f);
            }
            *reinterpret_cast<Vec<T, V> *>(h + (t + r) * hs.row) = out;
        }
    }
    if (final)
#pragma unroll
        for (int j = 0; j < V; ++j) final[i * a.dim + c + j] = state[j];
}

// A gradient's tensors.
template <class T>
struct ScanGrads {
    Seq<const T> dh, z, v, h;
    Seq<T> dz, dv;
    const float *d_final;
    float *d_initial;
};

template <class T, int V>
__global__ void __launch_bounds__(kWalkThreads) scan_walk_back_kernel(const ScanArgs a, const ScanGrads<T> g)
{
    const int64_t packs = a.dim / V, k = static_cast<int64_t>(blockIdx.x) * kWalkThreads + threadIdx.x;
    if (k >= a.batch * packs) return;
    const int64_t i = k / packs, c = (k - i * packs) * V, n = scan_length(a, i);
    using W = Vec<T, V>;
    auto at = [&](const Seq<const T> &s, int64_t t) { return *reinterpret_cast<const W *>(s.p + i * s.batch + t * s.row + c); };
    auto to = [&](const Seq<T> &s, int64_t t) -> W & { return *reinterpret_cast<W *>(s.p + i * s.batch + t * s.row + c); };
    W zero;
    float carry[V];  // f_{t+1} g_{t+1}
#pragma unroll
    for (int j = 0; j < V; ++j) carry[j] = g.d_final ? g.d_final[i * a.dim + c + j] : 0.0f, zero.x[j] = from_f32<T>(0.0f);
    for (int64_t t = a.length - 1; t >= 0; --t) {
        if (t >= n) {
            to(g.dz, t) = zero;
            to(g.dv, t) = zero;
            continue;
        }
        const W z = at(g.z, t), dh = at(g.dh, t), v = at(g.v, t), h = t ? at(g.h, t - 1) : zero;
        W dz, dv;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float before = t ? to_f32(h.x[j]) : a.initial ? a.initial[i * a.dim + c + j] : 0.0f;
            float f, shut;
            gate(to_f32(z.x[j]), f, shut);
            const float gt = __fadd_rn(to_f32(dh.x[j]), carry[j]), d = __fmul_rn(shut, gt);
            carry[j] = __fmul_rn(f, gt);
            dv.x[j] = from_f32<T>(d);
            dz.x[j] = from_f32<T>(__fmul_rn(__fmul_rn(f, d), __fsub_rn(before, to_f32(v.x[j]))));
        }
        to(g.dz, t) = dz;
        to(g.dv, t) = dv;
    }
    if (g.d_initial)
#pragma unroll
        for (int j = 0; j < V; ++j) g.d_initial[i * a.dim + c + j] = carry[j];
}

// ---------------------------------------------------------------------------------------------- tiles
// A thread's V columns are 16 bytes where rows allow it (a warp's lanes then cover 128-byte pieces of 4 rows), else one element
// (a warp covers 32 columns), and its rows 64 bytes of each tensor, or 16 elements.
template <class T, int V>
struct Tile {
    static constexpr int kLanes = V == 1 ? 32 : 8;            // lanes across a row
    static constexpr int kColumns = kLanes * V;
    static constexpr int kRows = V == 1 ? 16 : 4;             // of a thread
    static constexpr int kSegs = kTileThreads / kLanes;
    static constexpr int kChunk = kSegs * kRows;              // rows of a CTA in a step
    static constexpr bool kRing = V * sizeof(T) >= 4;         // what asynchronous copies can move
    static constexpr int kPack = V * sizeof(T);
};

// What a tile's CTA shares, behind its ring of copies.
template <int C>
struct TileShared {
    float2 warp[kTileWarps][C];           // each warp's composition
    float start[kTileWarps][C];           // the state that each warp starts with
    float2 rank[2][kMaxCluster][C];       // the CTAs' compositions, of this step and the last
};

template <int BYTES>
__device__ __forceinline__ void cp_async(void *dst, const void *src)
{
    if constexpr (BYTES == 16) cp_async16(dst, src);
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_addr(dst)), "l"(src), "n"(BYTES) : "memory");
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// A store to the shared memory of another CTA of the cluster, at the place that `p` is in this one.
__device__ __forceinline__ void store_remote(float2 *p, uint32_t rank, float2 v)
{
    uint32_t to;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_addr(p)), "r"(rank));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(v.x), "f"(v.y) : "memory");
}

// From each thread's composition (A, B) of its rows to the state that it starts with.  carry: in the first kColumns threads,
// the state before the step of this thread's column, and the one after it on return.
template <class L>
__device__ __forceinline__ void tile_start(float (&A)[L::kColumns / L::kLanes], float (&B)[L::kColumns / L::kLanes], float &carry,
                                           TileShared<L::kColumns> &sh, uint32_t rank, uint32_t ranks, int parity)
{
    constexpr int V = L::kColumns / L::kLanes;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = lane % L::kLanes * V;
#pragma unroll
    for (int o = L::kLanes; o < 32; o *= 2)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float a = __shfl_up_sync(0xffffffffu, A[j], o), b = __shfl_up_sync(0xffffffffu, B[j], o);
            if (lane >= o) {
                B[j] = __fmaf_rn(A[j], b, B[j]);
                A[j] = __fmul_rn(A[j], a);
            }
        }
    if (lane >= 32 - L::kLanes)
#pragma unroll
        for (int j = 0; j < V; ++j) sh.warp[warp][c0 + j] = make_float2(A[j], B[j]);
    if constexpr (L::kLanes < 32) {  // what the lanes before this one's make
#pragma unroll
        for (int j = 0; j < V; ++j) {
            A[j] = __shfl_up_sync(0xffffffffu, A[j], L::kLanes);
            B[j] = __shfl_up_sync(0xffffffffu, B[j], L::kLanes);
        }
    }
    if (lane < L::kLanes)
#pragma unroll
        for (int j = 0; j < V; ++j) A[j] = 1.0f, B[j] = 0.0f;
    __syncthreads();
    float2 before[kTileWarps], all = make_float2(1.0f, 0.0f);
    const bool column = threadIdx.x < L::kColumns;
    if (column) {
#pragma unroll
        for (int w = 0; w < kTileWarps; ++w) {
            const float2 x = sh.warp[w][threadIdx.x];
            before[w] = all;
            all = make_float2(__fmul_rn(x.x, all.x), __fmaf_rn(x.x, all.y, x.y));
        }
        if (ranks > 1)
            for (uint32_t r = 0; r < ranks; ++r) store_remote(&sh.rank[parity][rank][threadIdx.x], r, all);
    }
    if (ranks > 1) {
        cluster_arrive();
        cluster_wait();
    }
    if (column) {
        float mine = carry;
        if (ranks > 1) {
            float x = carry;
            for (uint32_t r = 0; r < ranks; ++r) {
                if (r == rank) mine = x;
                const float2 y = sh.rank[parity][r][threadIdx.x];
                x = __fmaf_rn(y.x, x, y.y);
            }
            carry = x;
        } else {
            carry = __fmaf_rn(all.x, carry, all.y);
        }
#pragma unroll
        for (int w = 0; w < kTileWarps; ++w) sh.start[w][threadIdx.x] = __fmaf_rn(before[w].x, mine, before[w].y);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) B[j] = __fmaf_rn(A[j], sh.start[warp][c0 + j], B[j]);
}

// blockIdx.x: tile of columns x sequence, in clusters along the rows (blockIdx.x / ranks is the tile).
template <class T, int V, int DEPTH>
__global__ void __launch_bounds__(kTileThreads) scan_tile_kernel(const ScanArgs a, const Seq<const T> zs, const Seq<const T> vs, const Seq<T> hs, float *final)
{
    using L = Tile<T, V>;
    using W = Vec<T, V>;
    constexpr int S = L::kRows;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ TileShared<L::kColumns> sh;
    const uint32_t rank = cluster_rank(), ranks = cluster_size();
    const uint32_t tile = blockIdx.x / ranks, tiles = static_cast<uint32_t>((a.dim + L::kColumns - 1) / L::kColumns);
    const int64_t i = tile / tiles, c0 = static_cast<int64_t>(tile % tiles) * L::kColumns;
    const int64_t c = c0 + threadIdx.x % L::kLanes * V;
    const bool inside = c < a.dim;
    const int64_t n = scan_length(a, i), stride = static_cast<int64_t>(ranks) * L::kChunk;
    const T *z = zs.p + i * zs.batch + c, *v = vs.p + i * vs.batch + c;
    T *h = hs.p + i * hs.batch + c;
    if (ranks > 1) cluster_arrive();  // every CTA runs before any stores into another
    const int64_t column = c0 + threadIdx.x;  // of the state that this thread carries
    const bool carries = threadIdx.x < L::kColumns && column < a.dim;
    float carry = carries && a.initial ? a.initial[i * a.dim + column] : 0.0f;
    const int64_t first = rank * static_cast<int64_t>(L::kChunk) + threadIdx.x / L::kLanes * S;  // this thread's first row
    W *ring = reinterpret_cast<W *>(smem) + threadIdx.x;  // a stage: S of z, then S of v, one per thread each
    auto fetch = [&](int64_t t, int stage) {
        if constexpr (L::kRing) {
#pragma unroll
            for (int r = 0; r < S; ++r)
                if (inside && t + r < n) {
                    cp_async<L::kPack>(ring + (stage * 2 * S + r) * kTileThreads, z + (t + r) * zs.row);
                    cp_async<L::kPack>(ring + ((stage * 2 + 1) * S + r) * kTileThreads, v + (t + r) * vs.row);
                }
            cp_async_commit();
        }
    };
    if constexpr (L::kRing)
        for (int d = 0; d < DEPTH; ++d) fetch(first + d * stride, d);
    if (ranks > 1) cluster_wait();
    int stage = 0, parity = 0;
    for (int64_t base = 0; base < a.length; base += stride) {
        const int64_t t = first + base;
        float f[S][V], u[S][V], A[V], B[V];
        W zv[S], vv[S];
        if constexpr (L::kRing) {
            cp_async_wait<DEPTH - 1>();
#pragma unroll
            for (int r = 0; r < S; ++r) {
                zv[r] = ring[(stage * 2 * S + r) * kTileThreads];
                vv[r] = ring[((stage * 2 + 1) * S + r) * kTileThreads];
            }
        } else {
#pragma unroll
            for (int r = 0; r < S; ++r)
                if (inside && t + r < n) {
                    zv[r] = *reinterpret_cast<const W *>(z + (t + r) * zs.row);
                    vv[r] = *reinterpret_cast<const W *>(v + (t + r) * vs.row);
                }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) A[j] = 1.0f, B[j] = 0.0f;
#pragma unroll
        for (int r = 0; r < S; ++r) {
            const bool on = inside && t + r < n;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float shut;
                gate(to_f32(zv[r].x[j]), f[r][j], shut);
                u[r][j] = on ? __fmul_rn(shut, to_f32(vv[r].x[j])) : 0.0f;
                f[r][j] = on ? f[r][j] : 1.0f;
                B[j] = __fmaf_rn(f[r][j], B[j], u[r][j]);
                A[j] = __fmul_rn(f[r][j], A[j]);
            }
        }
        if constexpr (L::kRing) fetch(t + DEPTH * stride, stage);
        tile_start<L>(A, B, carry, sh, rank, ranks, parity);
#pragma unroll
        for (int r = 0; r < S; ++r) {
            W out;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                B[j] = __fmaf_rn(f[r][j], B[j], u[r][j]);
                out.x[j] = from_f32<T>(t + r < n ? B[j] : 0.0f);
            }
            if (inside && t + r < a.length) *reinterpret_cast<W *>(h + (t + r) * hs.row) = out;
        }
        stage = stage + 1 == DEPTH ? 0 : stage + 1;
        parity ^= 1;
    }
    if (final && carries && rank == 0) final[i * a.dim + column] = carry;
}

// The same from the last row to the first: q counts rows from the end.
template <class T, int V, int DEPTH>
__global__ void __launch_bounds__(kTileThreads) scan_tile_back_kernel(const ScanArgs a, const ScanGrads<T> g)
{
    using L = Tile<T, V>;
    using W = Vec<T, V>;
    constexpr int S = L::kRows;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ TileShared<L::kColumns> sh;
    const uint32_t rank = cluster_rank(), ranks = cluster_size();
    const uint32_t tile = blockIdx.x / ranks, tiles = static_cast<uint32_t>((a.dim + L::kColumns - 1) / L::kColumns);
    const int64_t i = tile / tiles, c0 = static_cast<int64_t>(tile % tiles) * L::kColumns;
    const int64_t c = c0 + threadIdx.x % L::kLanes * V;
    const bool inside = c < a.dim;
    const int64_t n = scan_length(a, i), stride = static_cast<int64_t>(ranks) * L::kChunk, end = a.length - 1;
    const T *z = g.z.p + i * g.z.batch + c, *v = g.v.p + i * g.v.batch + c, *h = g.h.p + i * g.h.batch + c, *dh = g.dh.p + i * g.dh.batch + c;
    T *dz = g.dz.p + i * g.dz.batch + c, *dv = g.dv.p + i * g.dv.batch + c;
    if (ranks > 1) cluster_arrive();
    const int64_t column = c0 + threadIdx.x;
    const bool carries = threadIdx.x < L::kColumns && column < a.dim;
    float carry = carries && g.d_final ? g.d_final[i * a.dim + column] : 0.0f;
    const int64_t first = rank * static_cast<int64_t>(L::kChunk) + threadIdx.x / L::kLanes * S;
    W *ring = reinterpret_cast<W *>(smem) + threadIdx.x;  // a stage: S of z, of dh, of v and of h
    auto slot = [&](int stage, int what, int r) -> W & { return ring[((stage * 4 + what) * S + r) * kTileThreads]; };
    auto fetch = [&](int64_t q, int stage) {
        if constexpr (L::kRing) {
#pragma unroll
            for (int r = 0; r < S; ++r) {
                const int64_t t = end - q - r;
                if (inside && t >= 0 && t < n) {
                    cp_async<L::kPack>(&slot(stage, 0, r), z + t * g.z.row);
                    cp_async<L::kPack>(&slot(stage, 1, r), dh + t * g.dh.row);
                    cp_async<L::kPack>(&slot(stage, 2, r), v + t * g.v.row);
                    if (t) cp_async<L::kPack>(&slot(stage, 3, r), h + (t - 1) * g.h.row);
                }
            }
            cp_async_commit();
        }
    };
    if constexpr (L::kRing)
        for (int d = 0; d < DEPTH; ++d) fetch(first + d * stride, d);
    if (ranks > 1) cluster_wait();
    int stage = 0, parity = 0;
    for (int64_t base = 0; base < a.length; base += stride) {
        const int64_t q = first + base;
        float f[S][V], shut[S][V], A[V], B[V];
        W zr[L::kRing ? 1 : S], dr[L::kRing ? 1 : S], vr[L::kRing ? 1 : S], hr[L::kRing ? 1 : S];
        if constexpr (L::kRing) {
            cp_async_wait<DEPTH - 1>();
        } else {
#pragma unroll
            for (int r = 0; r < S; ++r) {
                const int64_t t = end - q - r;
                if (inside && t >= 0 && t < n) {
                    zr[r] = *reinterpret_cast<const W *>(z + t * g.z.row);
                    dr[r] = *reinterpret_cast<const W *>(dh + t * g.dh.row);
                    vr[r] = *reinterpret_cast<const W *>(v + t * g.v.row);
                    if (t) hr[r] = *reinterpret_cast<const W *>(h + (t - 1) * g.h.row);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) A[j] = 1.0f, B[j] = 0.0f;
#pragma unroll
        for (int r = 0; r < S; ++r) {
            const int64_t t = end - q - r;
            const bool on = inside && t >= 0 && t < n;
            W zv, d;
            if constexpr (L::kRing) zv = slot(stage, 0, r), d = slot(stage, 1, r);
            else zv = zr[r], d = dr[r];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                gate(to_f32(zv.x[j]), f[r][j], shut[r][j]);
                const float dht = on ? to_f32(d.x[j]) : 0.0f;
                f[r][j] = on ? f[r][j] : 1.0f;
                B[j] = __fmul_rn(f[r][j], __fadd_rn(dht, B[j]));
                A[j] = __fmul_rn(f[r][j], A[j]);
            }
        }
        tile_start<L>(A, B, carry, sh, rank, ranks, parity);
#pragma unroll
        for (int r = 0; r < S; ++r) {
            const int64_t t = end - q - r;
            const bool on = t < n;
            if (!inside || t < 0) continue;
            W d, vv, hv, oz, ov;
            if constexpr (L::kRing) d = slot(stage, 1, r), vv = slot(stage, 2, r), hv = slot(stage, 3, r);
            else d = dr[r], vv = vr[r], hv = hr[r];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float before = t ? to_f32(hv.x[j]) : a.initial ? a.initial[i * a.dim + c + j] : 0.0f;
                const float gt = __fadd_rn(to_f32(d.x[j]), B[j]), dvt = __fmul_rn(shut[r][j], gt);
                if (on) B[j] = __fmul_rn(f[r][j], gt);
                ov.x[j] = from_f32<T>(on ? dvt : 0.0f);
                oz.x[j] = from_f32<T>(on ? __fmul_rn(__fmul_rn(f[r][j], dvt), __fsub_rn(before, to_f32(vv.x[j]))) : 0.0f);
            }
            *reinterpret_cast<W *>(dz + t * g.dz.row) = oz;
            *reinterpret_cast<W *>(dv + t * g.dv.row) = ov;
        }
        if constexpr (L::kRing) fetch(q + DEPTH * stride, stage);
        stage = stage + 1 == DEPTH ? 0 : stage + 1;
        parity ^= 1;
    }
    if (g.d_initial && carries && rank == 0) g.d_initial[i * a.dim + column] = carry;
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
    a = ScanArgs{c->batch, c->length, s->cfg.dim, initial, lengths, c->length_type == EA_T_I64, s->status};
    return EA_OK;
}

constexpr int64_t kWalkRows = 16;  // sequences up to this length are walked along
constexpr int kDepth = 3, kBackDepth = 2;
constexpr int kTileCtasPerSm = 3;

// Launches a kernel of tiles: as many CTAs of a cluster along a sequence as it takes to fill the device, and no more than
// the sequence has chunks.
template <class L, class... KArgs, class... Args>
cudaError_t launch_tiles(const ea_scan *s, const ScanArgs &a, void (*kernel)(KArgs...), size_t smem, Args &&...args)
{
    const int64_t tiles = a.batch * over<int64_t>(a.dim, L::kColumns), chunks = over<int64_t>(a.length, L::kChunk);
    int ranks = 1;
    while (ranks < kMaxCluster && ranks < chunks && tiles * ranks < static_cast<int64_t>(s->dev.sms) * kTileCtasPerSm) ranks *= 2;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e == cudaSuccess && ranks > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    return launch_lm(kernel, dim3(static_cast<unsigned>(tiles * ranks)), kTileThreads, smem, s->stream, false, ranks, a, std::forward<Args>(args)...);
}

// f(std::integral_constant<int, V>) for the columns that an access of this call's tensors takes: 16 bytes of them or one.
template <class T, class F>
void with_columns(bool wide, F f)
{
    if (wide) f(std::integral_constant<int, 16 / sizeof(T)>());
    else f(std::integral_constant<int, 1>());
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
    if (a.batch && a.length) {
        if (r == EA_OK) r = check_address(z, c->type, "z");
        if (r == EA_OK) r = check_address(v, c->type, "v");
        if (r == EA_OK) r = check_address(h, c->type, "h");
        if (r == EA_OK) r = check_rows_apart(a.batch, a.length, c->h_batch, c->h_row, a.dim, "h");
    }
    if (r != EA_OK || !a.batch || (!a.length && !final)) return r;
    auto wide = [&](const void *p, int64_t batch, int64_t row) { return rows_on(16, p, c->type, a.dim, a.batch, a.length, batch, row); };
    const bool all = wide(z, c->z_batch, c->z_row) && wide(v, c->v_batch, c->v_row) && wide(h, c->h_batch, c->h_row);
    cudaError_t e = cudaSuccess;
    with_float(c->type, [&](auto *t) {
        using T = std::remove_reference_t<decltype(*t)>;
        const Seq<const T> zs{static_cast<const T *>(z), c->z_batch, c->z_row}, vs{static_cast<const T *>(v), c->v_batch, c->v_row};
        const Seq<T> hs{static_cast<T *>(h), c->h_batch, c->h_row};
        with_columns<T>(all, [&](auto columns) {
            constexpr int V = decltype(columns)::value;
            using L = Tile<T, V>;
            if (a.length <= kWalkRows) {
                const int64_t ctas = over<int64_t>(a.batch * (a.dim / V), kWalkThreads);
                scan_walk_kernel<T, V><<<static_cast<unsigned>(ctas), kWalkThreads, 0, s->stream>>>(a, zs, vs, hs, final);
                e = cudaGetLastError();
            } else {
                const size_t ring = L::kRing ? kDepth * 2 * L::kRows * kTileThreads * L::kPack : 0;
                e = launch_tiles<L>(s, a, scan_tile_kernel<T, V, kDepth>, ring, zs, vs, hs, final);
            }
        });
    });
    return lm_cuda(e, "launch");
}

int ea_scan_backward(ea_scan *s, const ea_scan_call *c, const void *dh, const void *z, const void *v, const void *h, const float *initial,
                     const void *lengths, const float *d_final, void *dz, void *dv, float *d_initial)
{
    ScanArgs a;
    int r = check_call(s, c, initial, lengths, a);
    if (r != EA_OK) return r;
    if (d_final) r = check_address(d_final, EA_T_F32, "d_final");
    if (r == EA_OK && d_initial) r = check_address(d_initial, EA_T_F32, "d_initial");
    if (a.batch && a.length) {
        const std::pair<const void *, const char *> all[] = {{dh, "dh"}, {z, "z"}, {v, "v"}, {h, "h"}, {dz, "dz"}, {dv, "dv"}};
        for (const auto &p : all)
            if (r == EA_OK) r = check_address(p.first, c->type, p.second);
        if (r == EA_OK) r = check_rows_apart(a.batch, a.length, c->dz_batch, c->dz_row, a.dim, "dz");
        if (r == EA_OK) r = check_rows_apart(a.batch, a.length, c->dv_batch, c->dv_row, a.dim, "dv");
        if (r == EA_OK && (dz == h || dv == h || dz == dv)) r = lm_fail(EA_E_INVAL, "dz and dv may be neither h nor one another");
    }
    if (r == EA_OK && d_initial && d_initial == initial) r = lm_fail(EA_E_INVAL, "d_initial may not be initial");
    if (r != EA_OK || !a.batch || (!a.length && !d_initial)) return r;
    auto wide = [&](const void *p, int64_t batch, int64_t row) { return rows_on(16, p, c->type, a.dim, a.batch, a.length, batch, row); };
    const bool all = wide(dh, c->dh_batch, c->dh_row) && wide(z, c->z_batch, c->z_row) && wide(v, c->v_batch, c->v_row) &&
                     wide(h, c->h_batch, c->h_row) && wide(dz, c->dz_batch, c->dz_row) && wide(dv, c->dv_batch, c->dv_row);
    cudaError_t e = cudaSuccess;
    with_float(c->type, [&](auto *t) {
        using T = std::remove_reference_t<decltype(*t)>;
        auto in = [](const void *p, int64_t batch, int64_t row) { return Seq<const T>{static_cast<const T *>(p), batch, row}; };
        auto out = [](void *p, int64_t batch, int64_t row) { return Seq<T>{static_cast<T *>(p), batch, row}; };
        const ScanGrads<T> g{in(dh, c->dh_batch, c->dh_row), in(z, c->z_batch, c->z_row),      in(v, c->v_batch, c->v_row), in(h, c->h_batch, c->h_row),
                             out(dz, c->dz_batch, c->dz_row), out(dv, c->dv_batch, c->dv_row), d_final,                     d_initial};
        with_columns<T>(all, [&](auto columns) {
            constexpr int V = decltype(columns)::value;
            using L = Tile<T, V>;
            if (a.length <= kWalkRows) {
                const int64_t ctas = over<int64_t>(a.batch * (a.dim / V), kWalkThreads);
                scan_walk_back_kernel<T, V><<<static_cast<unsigned>(ctas), kWalkThreads, 0, s->stream>>>(a, g);
                e = cudaGetLastError();
            } else {
                const size_t ring = L::kRing ? kBackDepth * 4 * L::kRows * kTileThreads * L::kPack : 0;
                e = launch_tiles<L>(s, a, scan_tile_back_kernel<T, V, kBackDepth>, ring, g);
            }
        });
    });
    return lm_cuda(e, "launch");
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
