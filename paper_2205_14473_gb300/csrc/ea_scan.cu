// ea_scan.cu -- ea_scan_forward and ea_scan_backward.
//
// Bound by HBM where the columns fill the device, else by a step's latency along each sequence.  One GB300, us a call, GB/s of the
// bytes that a call cannot do without, against a copy's 6,767:
//   16 x 1024 x 1600 bf16            26.5 us, 5,950 GB/s; its gradient 51.3 us, 6,130 GB/s
//   256 x 256 x 1024                 61.5 us, 6,550 GB/s;  320 x 256 x 1024 75.3 us, its gradient 148 us, 6,800 GB/s
//   2 x 65,536 x 1024                148 us, 5,430 GB/s (clusters of 8; 128 steps of 1.2 us)
//   9 sequences of up to 3001 x 515 binary32, off any boundary, gradient  54 us, 4,110 GB/s
//   1 x 65,536 x 128                 28 us (latency: 8 steps of clusters of 16, 128 CTAs in all)
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

constexpr float kMinusLog2e = -1.44269504088896340736f;

// 2^x and 1 / x by the hardware's approximations, within 2^-22 relative (x above 2^126 gives 0).
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float recip_fast(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// At most 126, so that neither 2^x nor its reciprocal leaves the normal numbers; NaN stays.
__device__ __forceinline__ float below_126(float x)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(126.0f));
    return r;
}

// V values of a thread's columns, in pairs where there are two or more.
template <int V>
struct Lanes {
    F2 x[V / 2];
    __device__ __forceinline__ void set(float a)
    {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) x[i] = both(a);
    }
    __device__ __forceinline__ void get(float (&y)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) unpack2(x[i], y[2 * i], y[2 * i + 1]);
    }
    __device__ __forceinline__ void put(const float (&y)[V])
    {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) x[i] = pack2(y[2 * i], y[2 * i + 1]);
    }
};
template <>
struct Lanes<1> {
    float x[1];
    __device__ __forceinline__ void set(float a) { x[0] = a; }
    __device__ __forceinline__ void get(float (&y)[1]) const { y[0] = x[0]; }
    __device__ __forceinline__ void put(const float (&y)[1]) { x[0] = y[0]; }
};
__device__ __forceinline__ float fma2(float a, float b, float c) { return __fmaf_rn(a, b, c); }
__device__ __forceinline__ float add2(float a, float b) { return __fadd_rn(a, b); }
__device__ __forceinline__ float times2(float a, float b) { return __fmul_rn(a, b); }
template <int V>
__device__ __forceinline__ Lanes<V> fma(const Lanes<V> &a, const Lanes<V> &b, const Lanes<V> &c)
{
    Lanes<V> r;
#pragma unroll
    for (int i = 0; i < (V + 1) / 2; ++i) r.x[i] = fma2(a.x[i], b.x[i], c.x[i]);
    return r;
}
template <int V>
__device__ __forceinline__ Lanes<V> operator*(const Lanes<V> &a, const Lanes<V> &b)
{
    Lanes<V> r;
#pragma unroll
    for (int i = 0; i < (V + 1) / 2; ++i) r.x[i] = times2(a.x[i], b.x[i]);
    return r;
}
template <int V>
__device__ __forceinline__ Lanes<V> operator+(const Lanes<V> &a, const Lanes<V> &b)
{
    Lanes<V> r;
#pragma unroll
    for (int i = 0; i < (V + 1) / 2; ++i) r.x[i] = add2(a.x[i], b.x[i]);
    return r;
}

// V consecutive elements in one access.
template <class T, int V>
struct alignas(V * sizeof(T)) Vec {
    T x[V];
};

template <class T, int V>
__device__ __forceinline__ Lanes<V> lanes(const Vec<T, V> &v)
{
    Lanes<V> r;
    float y[V];
    if constexpr (std::is_same<T, bf16>::value && V > 1) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(v.x);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) y[2 * i] = __uint_as_float(w[i] << 16), y[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else if constexpr (std::is_same<T, f16>::value && V > 1) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(v.x + 2 * i));
            y[2 * i] = p.x, y[2 * i + 1] = p.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = to_f32(v.x[i]);
    }
    r.put(y);
    return r;
}
template <class T, int V>
__device__ __forceinline__ Vec<T, V> rounded(const Lanes<V> &a)
{
    Vec<T, V> r;
    float y[V];
    a.get(y);
    if constexpr (std::is_same<T, bf16>::value && V > 1) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) *reinterpret_cast<__nv_bfloat162 *>(r.x + 2 * i) = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
    } else if constexpr (std::is_same<T, f16>::value && V > 1) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) *reinterpret_cast<__half2 *>(r.x + 2 * i) = __floats2half2_rn(y[2 * i], y[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r.x[i] = from_f32<T>(y[i]);
    }
    return r;
}
template <class T, int V>
__device__ __forceinline__ Vec<T, V> filled(float a)
{
    Lanes<V> x;
    x.set(a);
    return rounded<T, V>(x);
}

// V states, on a 16-byte boundary where V > 1.
template <int V>
__device__ __forceinline__ Lanes<V> load_states(const float *p)
{
    Lanes<V> r;
    alignas(16) float y[V];
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(y + i) = *reinterpret_cast<const float4 *>(p + i);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = p[i];
    }
    r.put(y);
    return r;
}
template <int V>
__device__ __forceinline__ void store_states(float *p, const Lanes<V> &a)
{
    alignas(16) float y[V];
    a.get(y);
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(p + i) = *reinterpret_cast<const float4 *>(y + i);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = y[i];
    }
}

// With e = 2^(-z log2 e), at most 2^126:  f = 1 / (1 + e) and 1 - f = e f.  In units of 2^-23, relative: e is off by 2 of the power of
// two and 0.61 |z| of its rounded exponent, f and 1 - f by no more than that (each has a factor below 1 for it) and 0.5 of the sum, 1
// of the reciprocal and 0.5 of the product: 4 + 0.7 |z|, where the smaller of the two is small, and less for the other.
// 2^-126 less makes f 0 where e is at its limit and does not change an f of 2^-101 or more.
template <int V>
__device__ __forceinline__ void gate(const Lanes<V> &z, Lanes<V> &f, Lanes<V> &shut)
{
    Lanes<V> scale, one, least, e;
    float y[V];
    scale.set(kMinusLog2e), one.set(1.0f), least.set(-0x1p-126f);
    (z * scale).get(y);
#pragma unroll
    for (int i = 0; i < V; ++i) y[i] = exp2_fast(below_126(y[i]));
    e.put(y);
    (e + one).get(y);
#pragma unroll
    for (int i = 0; i < V; ++i) y[i] = recip_fast(y[i]);
    f.put(y);
    shut = e * f;
    f = f + least;
}

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
    Lanes<V> state;
    state.set(0.0f);
    if (a.initial) state = load_states<V>(a.initial + i * a.dim + c);
    for (int64_t t = 0; t < a.length; t += kAhead) {
        Vec<T, V> zv[kAhead], vv[kAhead];
#pragma unroll
        for (int r = 0; r < kAhead; ++r)
            if (t + r < n) {
                zv[r] = *reinterpret_cast<const Vec<T, V> *>(z + (t + r) * zs.row);
                vv[r] = *reinterpret_cast<const Vec<T, V> *>(v + (t + r) * vs.row);
            }
#pragma unroll
        for (int r = 0; r < kAhead; ++r) {
            if (t + r >= a.length) break;
            if (t + r < n) {
                Lanes<V> f, shut;
                gate(lanes(zv[r]), f, shut);
                state = fma(f, state, shut * lanes(vv[r]));
            }
            *reinterpret_cast<Vec<T, V> *>(h + (t + r) * hs.row) = t + r < n ? rounded<T, V>(state) : filled<T, V>(0.0f);
        }
    }
    if (final) store_states(final + i * a.dim + c, state);
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
    const W zero = filled<T, V>(0.0f);
    Lanes<V> carry, minus, first;  // carry: f_{t+1} g_{t+1}
    carry.set(0.0f), minus.set(-1.0f), first.set(0.0f);
    if (g.d_final) carry = load_states<V>(g.d_final + i * a.dim + c);
    if (a.initial) first = load_states<V>(a.initial + i * a.dim + c);
    for (int64_t t = a.length - 1; t >= 0; --t) {
        if (t >= n) {
            to(g.dz, t) = zero;
            to(g.dv, t) = zero;
            continue;
        }
        const W z = at(g.z, t), dh = at(g.dh, t), v = at(g.v, t);
        const Lanes<V> before = t ? lanes(at(g.h, t - 1)) : first;
        Lanes<V> f, shut;
        gate(lanes(z), f, shut);
        const Lanes<V> gt = lanes(dh) + carry, d = shut * gt;
        carry = f * gt;
        to(g.dv, t) = rounded<T, V>(d);
        to(g.dz, t) = rounded<T, V>((f * d) * fma(lanes(v), minus, before));
    }
    if (g.d_initial) store_states(g.d_initial + i * a.dim + c, carry);
}

// ---------------------------------------------------------------------------------------------- tiles
// A thread's V columns are 16 bytes where rows allow it (eight lanes then cover a 128-byte piece of a row), else one element
// (a warp covers 32 columns).  S: its rows.  NT: threads of the CTA.  NARROW: two lanes of 16 bytes instead of eight.
template <class T, int V, int S, int NT, bool NARROW>
struct Tile {
    static constexpr int kThreads = NT;
    static constexpr int kLanes = V == 1 ? 32 : NARROW ? 2 : 8;  // lanes across a row
    static constexpr int kColumns = kLanes * V;
    static constexpr int kRows = S;
    static constexpr int kSegs = NT / kLanes;                 // threads along the rows
    static constexpr int kChunk = kSegs * kRows;              // rows of a CTA in a step
    static constexpr bool kRing = V > 1;                      // rows come through shared memory, else through registers
    static constexpr int kGroups = NT / kColumns;             // threads that compose a column's pieces, adjacent lanes
    static constexpr int kPieces = kSegs / kGroups;           // of each of them
    static constexpr int kTurn = V > 32 / kGroups ? V : 32 / kGroups;
};

// What a tile's CTA shares, behind its ring of copies.  A piece's columns are turned around by its group, kTurn of them (what a warp
// reads of a piece, and no less than a thread writes) for each, so that the lanes that read a column's pieces fall into different
// banks.
template <class L, bool CLUSTER>
struct TileShared {
    static constexpr int kRanks = CLUSTER ? kMaxCluster : 1;
    uint64_t arrived[2];                                       // barriers of `rank`
    float a[L::kSegs][L::kColumns], b[L::kSegs][L::kColumns];  // each thread's composition, then in b the state it starts with
    float2 rank[2][kRanks][L::kColumns];                       // the CTAs' compositions, of this step and the last
    static __device__ __forceinline__ int at(int seg, int column) { return column ^ (seg / L::kPieces * L::kTurn % L::kColumns); }
};

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
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Stores to the shared memory of a CTA of the cluster, at the place that `p` is in this one, and counts the 8 bytes on its
// barrier at the place that `bar` is.
__device__ __forceinline__ void store_remote(float2 *p, uint64_t *bar, uint32_t rank, float2 v)
{
    uint32_t to, at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_addr(p)), "r"(rank));
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(bar)), "r"(rank));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(to), "f"(v.x), "f"(v.y), "r"(at)
                 : "memory");
}

// A CTA's place in its cluster, and the step that its exchange is at.
struct Exchange {
    uint32_t rank = 0, ranks = 1, step = 0;
    bool late = false;  // whether a wait of this thread has run out

    template <class S>
    __device__ __forceinline__ void begin(S &sh)
    {
        rank = cluster_rank(), ranks = cluster_size();
        if (threadIdx.x == 0) {
            mbar_init(&sh.arrived[0], 1);
            mbar_init(&sh.arrived[1], 1);
            mbar_init_fence();
        }
        cluster_sync();  // before any CTA stores into another
    }

    // A column's composition, sent to all CTAs of the cluster by a group of G threads, into one of two buffers, and a wait for
    // theirs; returns the buffer that they are in.  A CTA sends the next but one after it has waited for the next, which the
    // others send after this one is read.  A thread whose wait has run out sends no more: the other CTAs' waits run out at
    // this step or the next then, and no barrier counts what belongs to a step that its CTA is not at.
    template <class S>
    __device__ __forceinline__ uint32_t pass(S &sh, float2 all, int column, int columns, int group, int G, uint32_t *status, long long limit = kWaitLimitCycles)
    {
        const uint32_t buffer = step & 1;
        if (!late) {
            if (threadIdx.x == 0) mbar_arrive_expect_tx(&sh.arrived[buffer], ranks * columns * 8);
            for (uint32_t r = group; r < ranks; r += G) store_remote(&sh.rank[buffer][rank][column], &sh.arrived[buffer], r, all);
            if (!mbar_wait<true>(&sh.arrived[buffer], step >> 1 & 1, limit)) {
                late = true;
                report_status(status, kStatusTimeout);
            }
        }
        ++step;
        return buffer;
    }

    // A CTA whose waits have all been completed is sent no more, and may end.  One with a wait that has run out stays until every
    // thread of the cluster has come here.
    __device__ __forceinline__ void end()
    {
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        if (late) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
};

template <int V>
__device__ __forceinline__ void to_shared(float *p, const Lanes<V> &a)
{
    store_states<V>(p, a);
}

// From each thread's composition (A, B) of its rows to the state that it starts with.  carry: the state before the step of
// column threadIdx.x / kGroups, and the one after it on return.  In a cluster the state before the first step is in the first
// CTA's hands alone, as part of what that makes of it: the same CTA writes the last state, which may lie in the same place.
template <bool CLUSTER, class L, int V>
__device__ __forceinline__ Lanes<V> tile_start(const Lanes<V> &A, const Lanes<V> &B, float &carry, TileShared<L, CLUSTER> &sh, Exchange &x, uint32_t *status)
{
    constexpr int G = L::kGroups;
    const int seg = threadIdx.x / L::kLanes, c0 = threadIdx.x % L::kLanes * V;
    const int column = threadIdx.x / G, group = threadIdx.x % G;
    to_shared(&sh.a[seg][sh.at(seg, c0)], A);
    to_shared(&sh.b[seg][sh.at(seg, c0)], B);
    __syncthreads();
    float pa[L::kPieces], pb[L::kPieces], m = 1.0f, y = 0.0f;  // what the pieces before each of the group's make of a state
#pragma unroll
    for (int k = 0; k < L::kPieces; ++k) {
        const int s = group * L::kPieces + k, at = sh.at(s, column);
        const float a = sh.a[s][at], b = sh.b[s][at];
        pa[k] = m, pb[k] = y;
        y = __fmaf_rn(a, y, b);
        m = __fmul_rn(a, m);
    }
#pragma unroll
    for (int o = 1; o < G; o *= 2) {  // the groups before this one's, and it
        const float a = __shfl_up_sync(0xffffffffu, m, o, G), b = __shfl_up_sync(0xffffffffu, y, o, G);
        if (group >= o) {
            y = __fmaf_rn(m, b, y);
            m = __fmul_rn(m, a);
        }
    }
    float2 all = make_float2(__shfl_sync(0xffffffffu, m, G - 1, G), __shfl_sync(0xffffffffu, y, G - 1, G));
    m = __shfl_up_sync(0xffffffffu, m, 1, G);
    y = __shfl_up_sync(0xffffffffu, y, 1, G);
    float state = carry;
    if constexpr (CLUSTER) {
        const bool first = x.step == 0 && x.rank == 0;
        if (first) all = make_float2(0.0f, __fmaf_rn(all.x, carry, all.y)), carry = 0.0f;
        const uint32_t buffer = x.pass(sh, all, column, L::kColumns, group, G, status);
        for (uint32_t r = 0; r < x.ranks; ++r) {
            if (r == x.rank && !first) state = carry;
            const float2 c = sh.rank[buffer][r][column];
            carry = __fmaf_rn(c.x, carry, c.y);
        }
    } else {
        carry = __fmaf_rn(all.x, carry, all.y);
    }
    if (group) state = __fmaf_rn(m, state, y);
#pragma unroll
    for (int k = 0; k < L::kPieces; ++k) {
        const int s = group * L::kPieces + k;
        sh.b[s][sh.at(s, column)] = __fmaf_rn(pa[k], state, pb[k]);
    }
    __syncthreads();
    return load_states<V>(&sh.b[seg][sh.at(seg, c0)]);
}

// blockIdx.x: sequence and tile of columns, in clusters along the rows (blockIdx.x / ranks is the tile).
template <class T, int V, int S, int NT, bool NARROW, int DEPTH, bool CLUSTER>
__global__ void __launch_bounds__(NT) scan_tile_kernel(const ScanArgs a, const Seq<const T> zs, const Seq<const T> vs, const Seq<T> hs, float *final)
{
    using L = Tile<T, V, S, NT, NARROW>;
    using W = Vec<T, V>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(16) TileShared<L, CLUSTER> sh;
    Exchange x;
    if constexpr (CLUSTER) x.begin(sh);
    const uint32_t tile = blockIdx.x / x.ranks, tiles = static_cast<uint32_t>((a.dim + L::kColumns - 1) / L::kColumns);
    const int64_t i = tile / tiles, c0 = static_cast<int64_t>(tile % tiles) * L::kColumns;
    const int64_t c = c0 + threadIdx.x % L::kLanes * V;
    const bool inside = c < a.dim;
    const int64_t n = scan_length(a, i), stride = static_cast<int64_t>(x.ranks) * L::kChunk;
    const int64_t column = c0 + threadIdx.x / L::kGroups;  // of the state that this thread carries
    float carry = column < a.dim && a.initial && x.rank == 0 ? a.initial[i * a.dim + column] : 0.0f;
    // This thread's first row of the step that is fetched, and of the step at hand, as rows that are left from there on.
    const int64_t first = x.rank * static_cast<int64_t>(L::kChunk) + threadIdx.x / L::kLanes * S;
    int next = static_cast<int>(n - first), left = next;
    const int step = static_cast<int>(stride);
    const T *z = zs.p + (i * zs.batch + first * zs.row + c), *v = vs.p + (i * vs.batch + first * vs.row + c);
    T *h = hs.p + (i * hs.batch + first * hs.row + c);
    // Rows that are not there have z of infinity and v of 0: the state passes through them.
    const W closed = filled<T, V>(__int_as_float(0x7f800000)), zero = filled<T, V>(0.0f);
    W *ring = reinterpret_cast<W *>(smem) + threadIdx.x;  // a stage: S of z, then S of v, one per thread each
    W zv[S], vv[S];
    auto fetch = [&](int stage) {
        const T *pz = z, *pv = v;
        W *to = ring + stage * (2 * S * NT);
#pragma unroll
        for (int r = 0; r < S; ++r, pz += zs.row, pv += vs.row) {
            const bool on = inside && next > r;
            if constexpr (L::kRing) {
                if (on) {
                    cp_async16(to + r * NT, pz);
                    cp_async16(to + (S + r) * NT, pv);
                } else {
                    to[r * NT] = closed;
                    to[(S + r) * NT] = zero;
                }
            } else {
                zv[r] = on ? *reinterpret_cast<const W *>(pz) : closed;
                vv[r] = on ? *reinterpret_cast<const W *>(pv) : zero;
            }
        }
        next -= step;
        z += stride * zs.row, v += stride * vs.row;
        if constexpr (L::kRing) cp_async_commit();
    };
    for (int d = 0; d < (L::kRing ? DEPTH : 1); ++d) fetch(d);
    int stage = 0;
    for (int64_t base = 0; base < n; base += stride) {
        if constexpr (L::kRing) {
            cp_async_wait<DEPTH - 1>();
            const W *from = ring + stage * (2 * S * NT);
#pragma unroll
            for (int r = 0; r < S; ++r) zv[r] = from[r * NT], vv[r] = from[(S + r) * NT];
        }
        Lanes<V> f[S], u[S], A, B;
#pragma unroll
        for (int r = 0; r < S; ++r) {
            Lanes<V> shut;
            gate(lanes(zv[r]), f[r], shut);
            u[r] = shut * lanes(vv[r]);
            B = r ? fma(f[r], B, u[r]) : u[r];
            A = r ? f[r] * A : f[r];
        }
        fetch(stage);
        Lanes<V> state = tile_start<CLUSTER>(A, B, carry, sh, x, a.status);
        T *to = h;
#pragma unroll
        for (int r = 0; r < S; ++r, to += hs.row) {
            state = fma(f[r], state, u[r]);
            if (inside && left > r) *reinterpret_cast<W *>(to) = rounded<T, V>(state);
        }
        left -= step;
        h += stride * hs.row;
        stage = stage + 1 == DEPTH ? 0 : stage + 1;
    }
    if (inside)
        for (int64_t t = n + x.rank * L::kSegs + threadIdx.x / L::kLanes; t < a.length; t += x.ranks * L::kSegs)
            *reinterpret_cast<W *>(hs.p + (i * hs.batch + t * hs.row + c)) = zero;
    if (final && column < a.dim && x.rank == 0 && threadIdx.x % L::kGroups == 0) final[i * a.dim + column] = carry;
    if constexpr (CLUSTER) x.end();
}

// The same from the sequence's last row to its first.
template <class T, int V, int S, int NT, bool NARROW, int DEPTH, bool CLUSTER>
__global__ void __launch_bounds__(NT) scan_tile_back_kernel(const ScanArgs a, const ScanGrads<T> g)
{
    using L = Tile<T, V, S, NT, NARROW>;
    using W = Vec<T, V>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(16) TileShared<L, CLUSTER> sh;
    Exchange x;
    if constexpr (CLUSTER) x.begin(sh);
    const uint32_t tile = blockIdx.x / x.ranks, tiles = static_cast<uint32_t>((a.dim + L::kColumns - 1) / L::kColumns);
    const int64_t i = tile / tiles, c0 = static_cast<int64_t>(tile % tiles) * L::kColumns;
    const int64_t c = c0 + threadIdx.x % L::kLanes * V;
    const bool inside = c < a.dim;
    const int64_t n = scan_length(a, i), stride = static_cast<int64_t>(x.ranks) * L::kChunk;
    const int64_t column = c0 + threadIdx.x / L::kGroups;
    float carry = column < a.dim && g.d_final && x.rank == 0 ? g.d_final[i * a.dim + column] : 0.0f;
    // Rows count from the end here: this thread's first ones of the step that is fetched and of the step at hand.
    const int64_t top = n - 1 - (x.rank * static_cast<int64_t>(L::kChunk) + threadIdx.x / L::kLanes * S);
    int next = static_cast<int>(top), t0 = next;
    const int step = static_cast<int>(stride);
    const T *z = g.z.p + (i * g.z.batch + top * g.z.row + c), *v = g.v.p + (i * g.v.batch + top * g.v.row + c);
    const T *dh = g.dh.p + (i * g.dh.batch + top * g.dh.row + c), *h = g.h.p + (i * g.h.batch + (top - 1) * g.h.row + c);
    T *dz = g.dz.p + (i * g.dz.batch + top * g.dz.row + c), *dv = g.dv.p + (i * g.dv.batch + top * g.dv.row + c);
    const W closed = filled<T, V>(__int_as_float(0x7f800000)), zero = filled<T, V>(0.0f);
    W *ring = reinterpret_cast<W *>(smem) + threadIdx.x;  // a stage: S of z, of dh, of v and of h
    auto slot = [&](int stage, int what, int r) -> W & { return ring[((stage * 4 + what) * S + r) * NT]; };
    constexpr int R = L::kRing ? 1 : S;
    W zr[R], dr[R], vr[R], hr[R], zn[R], dn[R], vn[R], hn[R];  // without the ring: this step's and the next one's
    auto fetch = [&](int stage) {
        const T *pz = z, *pd = dh, *pv = v, *ph = h;
#pragma unroll
        for (int r = 0; r < S; ++r) {
            const bool on = inside && next >= r;
            if constexpr (L::kRing) {
                if (on) {
                    cp_async16(&slot(stage, 0, r), pz);
                    cp_async16(&slot(stage, 1, r), pd);
                    cp_async16(&slot(stage, 2, r), pv);
                    if (next > r) cp_async16(&slot(stage, 3, r), ph);
                } else {
                    slot(stage, 0, r) = closed;
                    slot(stage, 1, r) = zero;
                }
            } else {
                zn[r] = on ? *reinterpret_cast<const W *>(pz) : closed;
                dn[r] = on ? *reinterpret_cast<const W *>(pd) : zero;
                vn[r] = on ? *reinterpret_cast<const W *>(pv) : zero;
                hn[r] = on && next > r ? *reinterpret_cast<const W *>(ph) : zero;
            }
            pz -= g.z.row, pd -= g.dh.row, pv -= g.v.row, ph -= g.h.row;
        }
        next -= step;
        z -= stride * g.z.row, dh -= stride * g.dh.row, v -= stride * g.v.row, h -= stride * g.h.row;
        if constexpr (L::kRing) cp_async_commit();
    };
    for (int d = 0; d < (L::kRing ? DEPTH : 1); ++d) fetch(d);
    Lanes<V> minus;
    minus.set(-1.0f);
    int stage = 0;
    for (int64_t base = 0; base < n; base += stride) {
        if constexpr (L::kRing) {
            cp_async_wait<DEPTH - 1>();
        } else {
#pragma unroll
            for (int r = 0; r < S; ++r) zr[r] = zn[r], dr[r] = dn[r], vr[r] = vn[r], hr[r] = hn[r];
            fetch(0);
        }
        Lanes<V> f[S], shut[S], A, B;
#pragma unroll
        for (int r = 0; r < S; ++r) {
            Lanes<V> d;
            if constexpr (L::kRing) gate(lanes(slot(stage, 0, r)), f[r], shut[r]), d = lanes(slot(stage, 1, r));
            else gate(lanes(zr[r]), f[r], shut[r]), d = lanes(dr[r]);
            B = f[r] * (r ? d + B : d);
            A = r ? f[r] * A : f[r];
        }
        Lanes<V> later = tile_start<CLUSTER>(A, B, carry, sh, x, a.status);
        T *pz = dz, *pv = dv;
#pragma unroll
        for (int r = 0; r < S; ++r, pz -= g.dz.row, pv -= g.dv.row)
            if (inside && t0 >= r) {
                W d, vv, hv;
                if constexpr (L::kRing) d = slot(stage, 1, r), vv = slot(stage, 2, r), hv = slot(stage, 3, r);
                else d = dr[r], vv = vr[r], hv = hr[r];
                Lanes<V> before = lanes(hv);
                if (t0 == r) {  // the sequence's first row
                    float y[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) y[j] = a.initial ? a.initial[i * a.dim + c + j] : 0.0f;
                    before.put(y);
                }
                const Lanes<V> gt = lanes(d) + later, dvt = shut[r] * gt;
                later = f[r] * gt;
                *reinterpret_cast<W *>(pv) = rounded<T, V>(dvt);
                *reinterpret_cast<W *>(pz) = rounded<T, V>((f[r] * dvt) * fma(lanes(vv), minus, before));
            }
        t0 -= step;
        dz -= stride * g.dz.row, dv -= stride * g.dv.row;
        if constexpr (L::kRing) fetch(stage);
        stage = stage + 1 == DEPTH ? 0 : stage + 1;
    }
    if (inside)
        for (int64_t t = n + x.rank * L::kSegs + threadIdx.x / L::kLanes; t < a.length; t += x.ranks * L::kSegs) {
            *reinterpret_cast<W *>(g.dz.p + (i * g.dz.batch + t * g.dz.row + c)) = zero;
            *reinterpret_cast<W *>(g.dv.p + (i * g.dv.batch + t * g.dv.row + c)) = zero;
        }
    if (g.d_initial && column < a.dim && x.rank == 0 && threadIdx.x % L::kGroups == 0) g.d_initial[i * a.dim + column] = carry;
    if constexpr (CLUSTER) x.end();
}

// ---------------------------------------------------------------------------------------------- self-test
constexpr int kTestRanks = 4, kTestSteps = 8, kTestColumns = 32;

struct TestShared {
    uint64_t arrived[2];
    float2 rank[2][kTestRanks][kTestColumns];
};

__device__ uint32_t g_exchange_status;

// One cluster whose CTAs exchange kTestSteps times.  CTA `silent` (-1: none) stops halfway, as one whose own wait has run out.
__global__ void __launch_bounds__(kWalkThreads) scan_exchange_kernel(long long limit, int silent)
{
    constexpr int G = kWalkThreads / kTestColumns;
    __shared__ __align__(16) TestShared sh;
    Exchange x;
    x.begin(sh);
    const int column = threadIdx.x / G;
    for (int t = 0; t < kTestSteps; ++t) {
        if (t == kTestSteps / 2 && static_cast<int>(x.rank) == silent) x.late = true;
        const float2 mine = make_float2(static_cast<float>(x.rank), static_cast<float>(t * kTestColumns + column));
        const uint32_t buffer = x.pass(sh, mine, column, kTestColumns, threadIdx.x % G, G, &g_exchange_status, limit);
        for (int r = 0; r < kTestRanks && !x.late; ++r) {
            const float2 c = sh.rank[buffer][r][column];
            if (c.x != static_cast<float>(r) || c.y != mine.y) report_status(&g_exchange_status, kStatusCheck);
        }
        __syncthreads();  // read before the next but one is sent
    }
    if (silent < 0 && x.rank == 0) x.late = true;  // stays until the others, who do not wait, have come to their end
    x.end();
}

}  // namespace ea

using namespace ea;

struct ea_scan {
    ea_scan_config cfg{};
    DeviceOf dev;
    cudaStream_t stream = nullptr;
    uint32_t *status = nullptr;
    Allowed allowed;
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

// Sequences up to kWalkRows are walked along; longer ones where so many 16-byte packs of columns are there to an SM that each
// thread's loads fill the device, and no longer than this: a tile's chunk of rows, and its exchange, costs the same whether its
// rows are there or not, and what it reads is further ahead.  bf16, us walked and in tiles:
//   up to 16 rows   400 x 16 x 1024 9.3 and 28.6;  64 x 16 x 1600 5.3 and 8.4, gradient 8.2 and 7.5, x 8 4.9 and 7.1.  Few of them would be
//     faster in tiles: 4 x 16 x 1600 5.3 and 2.5, gradient 7.8 and 2.6, x 4 2.5 and 2.5, 3.1 and 2.5
//   forward (4 rows of loads ahead)   320 x 33 x 1024 (270 packs) 18.2 and 24.6, x 48 0.95 of the tiles' time, x 64 1.12, x 256 113.7 and
//     75.4;  512 x 33 x 1024 (431 packs) 21.4 and 37.4, x 100 56.4 and 61.5, x 128 70.9 and 65.3;  256 x 64 x 1024 (215 packs) 1.27
//   gradient (none ahead)   320 x 33 x 1024 35.2 and 31.6, x 256 248 and 149;  400 x 33 x 1024 (337 packs) 0.97, x 40 44.9 and 40.3;
//     512 x 33 x 1024 41.8 and 47.8, x 40 50.1 and 49.9, x 64 77.5 and 58.8, x 256 296 and 236;  700 x 48 x 1024 (589 packs) 1.01;
//     1024 x 48 x 1024 (862 packs) 0.91, x 64 1.05, x 65 121.7 and 131.4, x 80 0.98, x 128 1.02;  in single elements 300 x 17 x 1025
//     (253 packs) 27.9 and 38.9, x 40 58.8 and 58.5, 320 x 48 x 1025 70.4 and 63.2
// That is where columns fill at least three quarters of their tiles; else any length is walked from kWalkPacks on: 45,600 x 300 x 8
// (an eighth, 300 packs) 183 and 679, gradient 418 and 1,111;  27,000 x 300 x 40 (0.62) 330 and 425, 723 and 724;  23,000 x 300 x 48 (0.75)
// 358 and 359, 757 and 604.
constexpr int64_t kWalkRows = 16, kWalkPacks = 256;
struct WalkRule {
    int64_t packs, rows;  // from so many packs an SM, up to so many rows
};
constexpr WalkRule kWalk[] = {{kWalkPacks, 48}, {400, 100}};
constexpr WalkRule kWalkBack[] = {{400, 40}, {600, 48}, {800, 80}}, kWalkBackOfOne[] = {{kWalkPacks, 40}, {600, 48}};
constexpr int64_t kFewRows = 512;  // a chunk of a narrow tile, forward
// Stages of a ring, and a thread's rows: 16-byte accesses without and within a cluster, and single elements.  Forward, 16 x 1024 x
// 1600 bf16: 26.6 us; 3 stages 27.8, 2 rows 32.0.  2 x 65,536 x 1024 in clusters: 148 us; 4 rows 171.  Gradient of the former: 51.3 us; 3
// stages 53.6, 4 rows 55.0, 1 row 59; in clusters (2 x 16,384 x 1024) 69.7 us; 2 rows 100, 8 rows 88.
constexpr int kDepth = 2, kTileThreads = 128;
constexpr int kRows = 4, kClusterRows = 8, kRowsOfOne = 8;
constexpr int kBackRows = 2, kBackClusterRows = 4, kBackRowsOfOne = 8;

// CTAs of a cluster along a sequence: 1 where the tiles alone occupy `fill` quarters of the SMs (an exchange costs as much as
// a step: 16 x 1024 x 1600 bf16 26.7 us without, 35.8 with clusters of two); else as many as that takes, in powers of two (8 x 2048 x
// 768: 24.4 us without, 21.5 of two, 23.2 of four;  a gradient of 9 x up to 3001 x 515, whose steps are longer, 62.7 of two and 52.7 of four,
// of full sequences 68.7 and 78.8), and no more than the sequence has chunks (a gradient of 1 x 1100 x 256, five chunks:
// 4.1 us of five, 5.3 of eight, three of which have no rows, 5.6 of four).  Clusters of 16 are for what occupies a part of the device even
// so (2 x 65,536 x 1024: 147.6 us in clusters of 8, 219 of 16, as not all of them fit at once).
template <class L>
int scan_ranks(const ea_scan *s, const ScanArgs &a, int fill)
{
    const int64_t tiles = a.batch * over<int64_t>(a.dim, L::kColumns), chunks = over<int64_t>(a.length, L::kChunk), sms = s->dev.sms;
    int ranks = 1;
    while (ranks < kMaxCluster && ranks < chunks && tiles * ranks * 4 < sms * fill && (ranks < 8 || tiles * 16 <= sms)) ranks *= 2;
    return static_cast<int>(std::min<int64_t>(ranks, std::max<int64_t>(chunks, 1)));
}

// Whether long sequences have so few columns that clusters of 16 leave SMs idle: tiles of a quarter of the columns then, whose
// CTAs take four times as many rows at a step (1 x 65,536 x 128 bf16 28 us instead of 62, its gradient 53 instead of 105;
// 1 x 4,096 x 64 4.4 instead of 5.7; 2 x 65,536 x 1024, with 32 wide tiles, 211 instead of 148).
template <class L>
bool few_tiles(const ea_scan *s, const ScanArgs &a)
{
    return a.length > kFewRows && a.batch * over<int64_t>(a.dim, L::kColumns) * kMaxCluster <= s->dev.sms;
}

template <class L, class... KArgs, class... Args>
cudaError_t launch_tiles(ea_scan *s, const ScanArgs &a, int ranks, int stages, void (*kernel)(KArgs...), Args &&...args)
{
    const size_t ring = L::kRing ? static_cast<size_t>(stages) * L::kRows * L::kThreads * 16 : 0;
    const cudaError_t e = s->allowed(kernel, ring, ranks > 1);
    if (e != cudaSuccess) return e;
    const int64_t tiles = a.batch * over<int64_t>(a.dim, L::kColumns);
    return launch_lm(kernel, dim3(static_cast<unsigned>(tiles * ranks)), L::kThreads, ring, s->stream, false, ranks, a, std::forward<Args>(args)...);
}

// whole: whether the call's tensors are read in 16-byte accesses.
template <size_t N>
bool walks(const ea_scan *s, const ScanArgs &a, int32_t type, bool whole, const WalkRule (&rules)[N])
{
    if (a.length <= kWalkRows) return true;
    const int64_t size = type_bytes(type), columns = whole ? 8 * 16 / size : 32;
    const bool full = 4 * a.dim >= 3 * over(a.dim, columns) * columns;
    const int64_t packs = a.batch * a.dim * size / (static_cast<int64_t>(s->dev.sms) * 16);
    if (!full) return packs >= kWalkPacks;
    return std::any_of(rules, rules + N, [&](const WalkRule &r) { return packs >= r.packs && a.length <= r.rows; });
}

bool states_on_16(const void *p, const void *q) { return (reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q)) % 16 == 0; }

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
    const bool whole = wide(z, c->z_batch, c->z_row) && wide(v, c->v_batch, c->v_row) && wide(h, c->h_batch, c->h_row);
    const bool walk = walks(s, a, c->type, whole, kWalk), all = whole && (!walk || states_on_16(initial, final));
    cudaError_t e = cudaSuccess;
    with_float(c->type, [&](auto *t) {
        using T = std::remove_reference_t<decltype(*t)>;
        const Seq<const T> zs{static_cast<const T *>(z), c->z_batch, c->z_row}, vs{static_cast<const T *>(v), c->v_batch, c->v_row};
        const Seq<T> hs{static_cast<T *>(h), c->h_batch, c->h_row};
        with_columns<T>(all, [&](auto columns) {
            constexpr int V = decltype(columns)::value;
            constexpr int S = V == 1 ? kRowsOfOne : kRows, SC = V == 1 ? kRowsOfOne : kClusterRows;
            using L = Tile<T, V, S, kTileThreads, false>;
            using LC = Tile<T, V, SC, kTileThreads, false>;
            using LN = Tile<T, V, SC, kTileThreads, (V > 1)>;
            if (walk) {
                const int64_t ctas = over<int64_t>(a.batch * (a.dim / V), kWalkThreads);
                scan_walk_kernel<T, V><<<static_cast<unsigned>(ctas), kWalkThreads, 0, s->stream>>>(a, zs, vs, hs, final);
                e = cudaGetLastError();
            } else {
                const int ranks = scan_ranks<LC>(s, a, 5);
                if (V > 1 && few_tiles<LC>(s, a))
                    e = launch_tiles<LN>(s, a, scan_ranks<LN>(s, a, 5), kDepth * 2, scan_tile_kernel<T, V, SC, kTileThreads, (V > 1), kDepth, true>, zs, vs, hs, final);
                else if (ranks > 1) e = launch_tiles<LC>(s, a, ranks, kDepth * 2, scan_tile_kernel<T, V, SC, kTileThreads, false, kDepth, true>, zs, vs, hs, final);
                else e = launch_tiles<L>(s, a, 1, kDepth * 2, scan_tile_kernel<T, V, S, kTileThreads, false, kDepth, false>, zs, vs, hs, final);
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
    const bool whole = wide(dh, c->dh_batch, c->dh_row) && wide(z, c->z_batch, c->z_row) && wide(v, c->v_batch, c->v_row) &&
                       wide(h, c->h_batch, c->h_row) && wide(dz, c->dz_batch, c->dz_row) && wide(dv, c->dv_batch, c->dv_row);
    const bool walk = whole ? walks(s, a, c->type, true, kWalkBack) : walks(s, a, c->type, false, kWalkBackOfOne);
    const bool all = whole && (!walk || (states_on_16(initial, d_final) && states_on_16(d_initial, nullptr)));
    cudaError_t e = cudaSuccess;
    with_float(c->type, [&](auto *t) {
        using T = std::remove_reference_t<decltype(*t)>;
        auto in = [](const void *p, int64_t batch, int64_t row) { return Seq<const T>{static_cast<const T *>(p), batch, row}; };
        auto out = [](void *p, int64_t batch, int64_t row) { return Seq<T>{static_cast<T *>(p), batch, row}; };
        const ScanGrads<T> g{in(dh, c->dh_batch, c->dh_row), in(z, c->z_batch, c->z_row),      in(v, c->v_batch, c->v_row), in(h, c->h_batch, c->h_row),
                             out(dz, c->dz_batch, c->dz_row), out(dv, c->dv_batch, c->dv_row), d_final,                     d_initial};
        with_columns<T>(all, [&](auto columns) {
            constexpr int V = decltype(columns)::value;
            constexpr int S = V == 1 ? kBackRowsOfOne : kBackRows, SC = V == 1 ? kBackRowsOfOne : kBackClusterRows;
            using L = Tile<T, V, S, kTileThreads, false>;
            using LC = Tile<T, V, SC, kTileThreads, false>;
            using LN = Tile<T, V, SC, kTileThreads, (V > 1)>;
            if (walk) {
                const int64_t ctas = over<int64_t>(a.batch * (a.dim / V), kWalkThreads);
                scan_walk_back_kernel<T, V><<<static_cast<unsigned>(ctas), kWalkThreads, 0, s->stream>>>(a, g);
                e = cudaGetLastError();
            } else {
                const int ranks = scan_ranks<LC>(s, a, 9);
                if (V > 1 && few_tiles<LC>(s, a))
                    e = launch_tiles<LN>(s, a, scan_ranks<LN>(s, a, 9), kDepth * 4, scan_tile_back_kernel<T, V, SC, kTileThreads, (V > 1), kDepth, true>, g);
                else if (ranks > 1) e = launch_tiles<LC>(s, a, ranks, kDepth * 4, scan_tile_back_kernel<T, V, SC, kTileThreads, false, kDepth, true>, g);
                else e = launch_tiles<L>(s, a, 1, kDepth * 4, scan_tile_back_kernel<T, V, S, kTileThreads, false, kDepth, false>, g);
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
    if (st & kStatusTimeout) return lm_fail(EA_E_TIMEOUT, "a wait within a cluster ran out");
    if (st & kStatusLength) return lm_fail(EA_E_DEVICE_CHECK, "a sequence's length lay outside its rows");
    return EA_OK;
}

int ea_scan_selftest_exchange(int64_t limit_cycles, int32_t silent, void *stream, int32_t *timed_out)
{
    if (!timed_out) return lm_fail(EA_E_INVAL, "timed_out is NULL");
    if (limit_cycles < 1 || limit_cycles > kWaitLimitCycles)
        return lm_fail(EA_E_INVAL, "limit_cycles must be in [1, %lld]", static_cast<long long>(kWaitLimitCycles));
    if (silent < -1 || silent >= kTestRanks) return lm_fail(EA_E_INVAL, "silent is a CTA, or -1 for none");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uint32_t zero = 0;
    uint32_t st = 0;
    cudaError_t e = cudaMemcpyToSymbolAsync(g_exchange_status, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess)
        e = launch_lm(scan_exchange_kernel, dim3(kTestRanks), kWalkThreads, 0, s, false, kTestRanks, static_cast<long long>(limit_cycles), static_cast<int>(silent));
    if (e == cudaSuccess) e = cudaMemcpyFromSymbolAsync(&st, g_exchange_status, sizeof st, 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) return lm_cuda(e, "exchange self-test");
    if (st & kStatusCheck) return lm_fail(EA_E_DEVICE_CHECK, "an exchange delivered other values than were sent");
    *timed_out = st & kStatusTimeout ? 1 : 0;
    return EA_OK;
}

int ea_scan_destroy(ea_scan *s)
{
    delete s;
    return EA_OK;
}

}  // extern "C"
