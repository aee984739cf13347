// ea_embed.cu -- the lookup of tokens in an embedding table (ea_embed_lookup) and the gradient of the table
// (ea_embed_grad).
//
// Both move rows and do next to no arithmetic.  Measured on one GB300 (us a call, calls one behind another; GB/s of the
// bytes that a call cannot do without, against a copy's 6,800):
//   lookup, 16,384 of 50,257 x 1600, 32 to 16 bits   19.2 us, 4,840 GB/s (a plain copy of as many bytes: 25.8 us)
//     the table off a 16-byte boundary, or 1601 wide 24.8 us
//   gradient of that batch, 32 bits written          85 us, 4,400 GB/s: the sort and the zero rows (52 us), sums, joins
//     added to a tied one                            56 us
//     the table off a 16-byte boundary, or 1601 wide 99 us
//   gradient, 260,096 tokens, 768 wide, half padding 94 us, 3,140 GB/s: six launches of sort (38 us), sums (41; 4.7 TB/s)
//     the table off a 16-byte boundary, or 769 wide  143, 159 us
#include <cooperative_groups.h>
#include <type_traits>

#include "ea_async.cuh"
#include "ea_lm.cuh"

namespace ea {

constexpr uint32_t kStatusToken = 4u;  // a token outside the table

struct EmbedArgs {
    int64_t n;                   // tokens
    uint32_t inner, magic;       // tokens per row of the batch (0: all in one row), and t / inner = t * magic >> 32 + shift
    int shift;
    int64_t token_outer, token_inner, row_outer, row_inner, table_stride;
    int64_t vocab, dim, padding;
    float scale;
    int token64;
    const void *tokens;
    uint32_t *status;
};

// Token t of the call lies in row i = t / inner of the batch.  The division of t < 2^30 by the constant inner >= 2
// is a multiplication (Granlund and Montgomery, "Division by invariant integers using multiplication"): with
// s = ceil(log2 inner) and magic = floor(2^(31 + s) / inner) + 1 < 2^32 the error stays below 1 / inner.
__device__ __forceinline__ uint32_t batch_row(const EmbedArgs &a, uint32_t t)
{
    return a.inner ? __umulhi(t, a.magic) >> a.shift : 0;
}

__device__ __forceinline__ int64_t token_at(const EmbedArgs &a, uint32_t t)
{
    const uint32_t i = batch_row(a, t);
    const int64_t at = i * a.token_outer + static_cast<int64_t>(t - i * a.inner) * a.token_inner;
    return a.token64 ? static_cast<const int64_t *>(a.tokens)[at] : static_cast<const int32_t *>(a.tokens)[at];
}

__device__ __forceinline__ int64_t row_at(const EmbedArgs &a, uint32_t t)
{
    const uint32_t i = batch_row(a, t);
    return i * a.row_outer + static_cast<int64_t>(t - i * a.inner) * a.row_inner;
}

// VEC consecutive elements, moved in words of up to 16 bytes (to which their address is aligned).
template <class Y, int VEC>
struct alignas(VEC * sizeof(Y) > 16 ? 16 : VEC * sizeof(Y)) Pack {
    Y y[VEC];
};
template <class Y, int VEC, bool STORE>
__device__ __forceinline__ void move_pack(Y *p, Pack<Y, VEC> &x)
{
    using Word = typename std::conditional<sizeof(x) >= 16, uint4, typename std::conditional<sizeof(x) == 8, uint2, Pack<Y, VEC>>::type>::type;
#pragma unroll
    for (int k = 0; k < static_cast<int>(sizeof(x) / sizeof(Word)); ++k) {
        if (STORE) reinterpret_cast<Word *>(p)[k] = reinterpret_cast<const Word *>(&x)[k];
        else reinterpret_cast<Word *>(&x)[k] = reinterpret_cast<const Word *>(p)[k];
    }
}
template <class Y, int VEC>
__device__ __forceinline__ void load_pack(const Y *p, Pack<Y, VEC> &x) { move_pack<Y, VEC, false>(const_cast<Y *>(p), x); }
template <class Y, int VEC>
__device__ __forceinline__ void store_pack(Y *p, Pack<Y, VEC> &x) { move_pack<Y, VEC, true>(p, x); }

// ------------------------------------------------------------------------------------------- lookup
//
// A copy of rows: a row is packs of 16 bytes of the table (single elements where an address or the width is not a
// multiple of that), several per thread, all of its loads in flight together.
//   rows of kWideRow packs or more: a warp takes a piece of one row, so that its addresses are formed once for all of
//     its packs; one token's row is still spread over as many warps as it has pieces;
//   narrower ones: the packs of all tokens are dealt out in order, so that no lane idles.
// The index arithmetic decides: dealt out in order, 16,384 rows of 400 packs took 23.8 us; a piece per warp takes 19.2.  In
// 16 bits, dealt out or by pieces: 48 packs 6.4 and 7.0 us, 64 packs 8.2 either way, 96 10.5 and 10.2, 127 14.4 and 12.3.

constexpr int kLookupThreads = 256;
constexpr int kLookupUnroll = 4;  // narrow rows
constexpr int kWideUnroll = 8;
constexpr int kWideRow = 64;
constexpr int kLookupCtasPerSm = 4;

struct LookupArgs {
    EmbedArgs e;
    uint32_t packs, magic;  // per row; quotient by it, as in batch_row (packs >= 2)
    int shift;
    int64_t total;          // of all tokens
    uint32_t turn_rows, turn_packs;  // rows and packs over from one turn of a CTA to its next
};

template <class W, class Y, int VEC>
__global__ void __launch_bounds__(kLookupThreads) lookup_narrow_kernel(const LookupArgs a, const W *w, Y *y)
{
    constexpr int kSpan = kLookupThreads * kLookupUnroll;  // packs of a turn
    __shared__ int64_t from[2][kSpan + 1], to[2][kSpan + 1];  // a turn's rows, in elements from w (-1: none) and y
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kSpan;
    auto quotient = [&](uint32_t i) { return a.packs > 1 ? __umulhi(i, a.magic) >> a.shift : i; };
    // pack `at` is the skip-th of token row0 (a 64-bit division costs as much as ten packs)
    const int64_t start = static_cast<int64_t>(blockIdx.x) * kSpan;
    uint32_t row0 = a.total < (1 << 30) ? quotient(static_cast<uint32_t>(start)) : static_cast<uint32_t>(start / a.packs);
    uint32_t skip = static_cast<uint32_t>(start - static_cast<int64_t>(row0) * a.packs);
    auto look = [&](int64_t at, int turn) {
        const uint32_t rows = quotient(skip + static_cast<uint32_t>(min(a.total - at, static_cast<int64_t>(kSpan))) - 1) + 1;
        for (uint32_t r = threadIdx.x; r < rows; r += kLookupThreads) {
            const uint32_t t = row0 + r;
            const int64_t v = token_at(a.e, t);
            const bool inside = v >= 0 && v < a.e.vocab;
            if (!inside) atomicOr(a.e.status, kStatusToken);
            from[turn][r] = inside ? v * a.e.table_stride : -1;
            to[turn][r] = row_at(a.e, t);
        }
    };
    int turn = 0;
    look(start, 0);
    __syncthreads();
    for (int64_t at = start; at < a.total; at += stride) {
        const uint32_t n = static_cast<uint32_t>(min(a.total - at, static_cast<int64_t>(kSpan)));
        Pack<W, VEC> x[kLookupUnroll];
        Y *dst[kLookupUnroll];
        bool inside[kLookupUnroll];
#pragma unroll
        for (int k = 0; k < kLookupUnroll; ++k) {
            const uint32_t i = k * kLookupThreads + threadIdx.x;
            dst[k] = nullptr;
            if (i >= n) continue;
            const uint32_t r = quotient(skip + i), j = (skip + i - r * a.packs) * VEC;
            dst[k] = y + to[turn][r] + j;
            inside[k] = from[turn][r] >= 0;
            if (inside[k]) load_pack<W, VEC>(w + from[turn][r] + j, x[k]);
        }
        turn ^= 1;
        row0 += a.turn_rows;
        skip += a.turn_packs;
        if (skip >= a.packs) {
            skip -= a.packs;
            ++row0;
        }
        if (at + stride < a.total) look(at + stride, turn);  // the next turn's tokens, while these rows are on their way
#pragma unroll
        for (int k = 0; k < kLookupUnroll; ++k) {
            if (!dst[k]) continue;
            Pack<Y, VEC> out;
#pragma unroll
            for (int i = 0; i < VEC; ++i) out.y[i] = from_f32<Y>(inside[k] ? __fmul_rn(to_f32(x[k].y[i]), a.e.scale) : 0.0f);
            store_pack<Y, VEC>(dst[k], out);
        }
        __syncthreads();
    }
}

struct LookupWideArgs {
    EmbedArgs e;
    uint32_t packs, piece, pieces;     // of a row; of a piece; pieces of a row
    uint32_t turn_rows, turn_pieces;   // rows and pieces over from one turn of a warp to its next
    int64_t total;                     // pieces of all tokens
};

template <class W, class Y, int VEC>
__global__ void __launch_bounds__(kLookupThreads, kLookupCtasPerSm) lookup_wide_kernel(const LookupWideArgs a, const W *w, Y *y)
{
    const int lane = threadIdx.x & 31;
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kLookupThreads / 32);
    const int64_t start = static_cast<int64_t>(blockIdx.x) * (kLookupThreads / 32) + (threadIdx.x >> 5);
    if (start >= a.total) return;
    uint32_t t = static_cast<uint32_t>(a.pieces == 1 ? start : start / a.pieces);
    uint32_t c = static_cast<uint32_t>(start - static_cast<int64_t>(t) * a.pieces);
    int64_t v = token_at(a.e, t);
    for (int64_t u = start; u < a.total; u += warps) {
        const bool inside = v >= 0 && v < a.e.vocab;
        if (!inside && c == 0 && lane == 0) atomicOr(a.e.status, kStatusToken);
        const uint32_t p0 = c * a.piece, n = min(a.piece, a.packs - p0);
        const W *from = w + (inside ? v : 0) * a.e.table_stride + (p0 + lane) * VEC;
        Y *to = y + row_at(a.e, t) + (p0 + lane) * VEC;
        Pack<W, VEC> x[kWideUnroll];
#pragma unroll
        for (int k = 0; k < kWideUnroll; ++k)
            if (inside && 32 * k + lane < n) load_pack<W, VEC>(from + 32 * k * VEC, x[k]);
            else x[k] = Pack<W, VEC>{};
        t += a.turn_rows;
        c += a.turn_pieces;
        if (c >= a.pieces) {
            c -= a.pieces;
            ++t;
        }
        if (u + warps < a.total) v = token_at(a.e, t);  // the next turn's token, while this row is on its way
#pragma unroll
        for (int k = 0; k < kWideUnroll; ++k) {
            if (32 * k + lane >= n) break;
            Pack<Y, VEC> out;
#pragma unroll
            for (int i = 0; i < VEC; ++i) out.y[i] = from_f32<Y>(__fmul_rn(to_f32(x[k].y[i]), inside ? a.e.scale : 0.0f));
            store_pack<Y, VEC>(to + 32 * k * VEC, out);
        }
    }
}

// ------------------------------------------------------------------------------- the table's gradient
//
// dw[v] = scale * sum of dy[t] over the t with token v: a sum over equal keys.  Tokens are sorted with their
// positions (stable, so that each sum runs in the order of the positions), the sorted list is cut into chunks
// of equal length, and a CTA sums a chunk's rows, one accumulator per column in registers, and stores a row of
// dw wherever the token changes.  A token whose run crosses a chunk's border leaves a binary32 partial sum per
// chunk instead, and combine_kernel adds those in the chunks' order.  So every row of dy is read once, a long
// run (the tokens of a natural text are a few thousand times more frequent at the top than at the bottom) is
// split over as many CTAs as its length asks for, and the result is a function of the inputs alone.
//
//   up to kClusterTokens   order_kernel: one cluster of CTAs sorts in shared memory, exchanging digit counts and
//                          keys through distributed shared memory, while the other CTAs write the zero rows of
//                          the tokens that do not occur (those need no order, only the set of tokens);
//   more                   hist, scan and scatter launches per digit; the first marks the tokens in a bitmap, and
//                          the others, none of which fills the GPU, write a share of the zero rows each;
//   then                   sum_kernel, combine_kernel.

constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kDigits = 256;                 // of one radix pass
constexpr int kCluster = 8;                  // CTAs that sort together
constexpr int kMaxItems = 16;                // keys per thread of a sorting CTA
// CTAs per SM that write zero rows beside it: 16,384 tokens of 50,257 x 1600 85.3 us, with two of them 95.2, with four 85.5;
// 16-bit rows 1024 wide 47.0, 47.3 and 48.8.
constexpr int kZeroCtasPerSm = 3;
// One CTA or a cluster, tokens of 30,522 x 768: overwritten, 1,024 tokens 29.2 and 30.6 us, 2,048 29.4 and 30.7, 4,096 32.9
// and 32.0; added to what is there, where the sort is all of the first launch, 16.4 each, 20.5 and 17.4, 26.7 and 18.8.
constexpr int kOneCtaTokens = kSortThreads * 4;
// A cluster or the longer sorts, tokens of 50,257 x 1024: 16,384 64 and 85 us, 32,768 81 and 91, 40,000 106 and 93, 65,536
// 139 and 103; added to what is there 46 and 51, 69 and 68, 89 and 73, 110 and 95.  It is as many as a cluster holds; above
// 32,768, where a CTA's 16 keys per thread leave room for no second one on an SM, the longer sorts would be faster.
constexpr int kClusterTokens = kSortThreads * kMaxItems * kCluster;
constexpr int kTileItems = 2;                // keys per thread of a tile of the longer sorts
constexpr int kTile1 = kSortThreads * kTileItems;

struct SortArgs {
    EmbedArgs e;
    uint32_t *key, *pos;       // the sorted list
    int passes, bits;          // radix passes of `bits` bits each; keys are 0 .. vocab
};

// Key of token t: the token, or vocab (which sorts last and is ignored) where it takes no gradient.
__device__ __forceinline__ uint32_t key_at(const EmbedArgs &a, uint32_t t, bool report)
{
    const int64_t v = token_at(a, t);
    const bool inside = v >= 0 && v < a.vocab;
    if (report && !inside) atomicOr(a.status, kStatusToken);
    return static_cast<uint32_t>(inside && v != a.padding ? v : a.vocab);
}

// Ranks of a CTA's keys within their digit.  Warp w holds the kSortThreads / 32 * ITEMS slots from w * 32 * ITEMS
// on, slot 32 i + lane in item i.  On return rank[i] counts the equal digits before it in its warp, and
// hist[w][d] those of the warps before; total[d] is the CTA's count.  Both are complete after the next barrier.
template <int ITEMS>
__device__ __forceinline__ void rank_digits(const uint32_t (&digit)[ITEMS], uint32_t (&rank)[ITEMS], uint32_t (*hist)[kDigits],
                                            uint32_t *total, int digits)
{
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int d = lane; d < digits; d += 32) hist[w][d] = 0;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t peers = __match_any_sync(0xffffffffu, digit[i]);
        const int leader = __ffs(peers) - 1;
        uint32_t before = 0;
        if (lane == leader) {
            before = hist[w][digit[i]];
            hist[w][digit[i]] = before + __popc(peers);
        }
        rank[i] = __shfl_sync(0xffffffffu, before, leader) + __popc(peers & ((1u << lane) - 1u));
        __syncwarp();
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads) {
        uint32_t sum = 0;
#pragma unroll
        for (int k = 0; k < kSortWarps; ++k) {
            const uint32_t n = hist[k][d];
            hist[k][d] = sum;
            sum += n;
        }
        total[d] = sum;
    }
}

// base[d] <- the sum of count over the smaller digits + add, for threads d < kDigits (count 0 above `digits`).
__device__ __forceinline__ void scan_digits(uint32_t count, uint32_t add, uint32_t *base, uint32_t *warp_sums)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    uint32_t sum = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += up;
    }
    if (threadIdx.x < kDigits && lane == 31) warp_sums[w] = sum;
    __syncthreads();
    if (threadIdx.x < kDigits) {
        for (int k = 0; k < w; ++k) sum += warp_sums[k];
        base[threadIdx.x] = sum - count + add;
    }
    __syncthreads();
}

// The table that zero rows are written to: all of its types have an all-zero 0.
struct ZeroTable {
    unsigned char *dw;
    int elem;  // bytes
};

// A row of `bytes` zeros (elements of 2 or 4 bytes), by one warp.
__device__ __forceinline__ void zero_row(unsigned char *p, int64_t bytes)
{
    const int lane = threadIdx.x & 31;
    const int64_t head = min(bytes, static_cast<int64_t>(-reinterpret_cast<uintptr_t>(p) & 15)), body = (bytes - head) / 16;
    uint4 *q = reinterpret_cast<uint4 *>(p + head);
    for (int64_t j = lane; j < body; j += 32) q[j] = make_uint4(0, 0, 0, 0);
    const int64_t tail = head + 16 * body;  // at most 15 bytes on either side
    const int64_t at = lane < 8 ? lane * 2 : tail + (lane - 8) * 2, end = lane < 8 ? head : bytes;
    if (lane < 16 && at < end) *reinterpret_cast<uint16_t *>(p + at) = 0;
}

// Zero rows of the tokens in [row0, row1) that do not occur.  mark(lo, hi, set) calls set(v) for every token v of
// [lo, hi) that does.
template <class Mark>
__device__ __forceinline__ void zero_rows(const EmbedArgs &a, const ZeroTable &z, int64_t row0, int64_t row1, uint32_t *bits,
                                          int64_t bit_words, Mark mark)
{
    const int w = threadIdx.x >> 5, warps = blockDim.x >> 5;
    for (int64_t lo = row0; lo < row1; lo += bit_words * 32) {
        const int64_t hi = min(row1, lo + bit_words * 32);
        const int64_t words = (hi - lo + 31) / 32;
        for (int64_t i = threadIdx.x; i < words; i += blockDim.x) bits[i] = 0;
        __syncthreads();
        mark(lo, hi, [&](int64_t v) {
            const uint32_t bit = 1u << ((v - lo) & 31);
            uint32_t &word = bits[(v - lo) >> 5];
            if (!(*static_cast<volatile uint32_t *>(&word) & bit)) atomicOr(&word, bit);
        });
        __syncthreads();
        for (int64_t v = lo + w; v < hi; v += warps)
            if (!(bits[(v - lo) >> 5] >> ((v - lo) & 31) & 1u))
                zero_row(z.dw + v * a.table_stride * z.elem, a.dim * z.elem);
        __syncthreads();
    }
}

// Shared memory of a sorting CTA: two buffers of its keys and positions, the warps' digit counts and the CTA's.
template <int ITEMS>
constexpr size_t kSortSmem = size_t{2} * ITEMS * kSortThreads * 8 + (kSortWarps * kDigits + 2 * kDigits + 32) * 4;

template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads) order_kernel(const SortArgs a, const ZeroTable z, int64_t rows_per_cta)
{
    namespace cg = cooperative_groups;
    pdl_trigger();
    extern __shared__ __align__(16) unsigned char smem[];
    cg::cluster_group cluster = cg::this_cluster();
    const unsigned ctas = cluster.num_blocks();
    const uint32_t n = static_cast<uint32_t>(a.e.n);
    if (blockIdx.x >= ctas) {  // not the sorting cluster: zero rows
        const int64_t row0 = static_cast<int64_t>(blockIdx.x - ctas) * rows_per_cta;
        zero_rows(a.e, z, row0, min(a.e.vocab, row0 + rows_per_cta), reinterpret_cast<uint32_t *>(smem),
                  static_cast<int64_t>(kSortSmem<ITEMS> / 4), [&](int64_t lo, int64_t hi, auto set) {
#pragma unroll 4
                      for (uint32_t t = threadIdx.x; t < n; t += kSortThreads) {
                          const int64_t v = token_at(a.e, t);
                          if (v >= lo && v < hi && v != a.e.padding) set(v);
                      }
                  });
        return;
    }
    constexpr uint32_t kKeys = ITEMS * kSortThreads;  // of a CTA
    uint2 *buf = reinterpret_cast<uint2 *>(smem);
    auto hist = reinterpret_cast<uint32_t(*)[kDigits]>(smem + size_t{2} * kKeys * 8);
    uint32_t *total = &hist[kSortWarps][0], *base = total + kDigits, *warp_sums = base + kDigits;
    const uint32_t me = cluster.block_rank(), slot0 = (threadIdx.x >> 5) * 32 * ITEMS + (threadIdx.x & 31);
    const int digits = 1 << a.bits;
    uint2 item[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {  // slots beyond the tokens sort last
        const uint32_t t = me * kKeys + slot0 + 32 * i;
        item[i] = make_uint2(t < n ? key_at(a.e, t, true) : 0xffffffffu, t);
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        uint32_t digit[ITEMS], rank[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) digit[i] = (item[i].x >> (pass * a.bits)) & (digits - 1);
        rank_digits(digit, rank, hist, total, digits);
        cluster.sync();  // every CTA's total
        uint32_t before = 0, all = 0;
        if (threadIdx.x < digits)
            for (unsigned c = 0; c < ctas; ++c) {
                const uint32_t m = cluster.map_shared_rank(total, c)[threadIdx.x];
                before += c < me ? m : 0;
                all += m;
            }
        scan_digits(all, before, base, warp_sums);
        const bool last = pass + 1 == a.passes;
        uint2 *to = buf + (pass & 1) * kKeys;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint32_t at = base[digit[i]] + hist[threadIdx.x >> 5][digit[i]] + rank[i];
            if (!last) {
                cluster.map_shared_rank(to, at / kKeys)[at % kKeys] = item[i];
            } else if (at < n) {
                a.key[at] = item[i].x;
                a.pos[at] = item[i].y;
            }
        }
        cluster.sync();  // every CTA's keys have arrived, and its total has been read
        if (!last)
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) item[i] = to[slot0 + 32 * i];
    }
}

// The longer sorts.  hist is digit-major: hist[d * tiles + tile].
struct TileSortArgs {
    EmbedArgs e;
    const uint32_t *key_in, *pos_in;  // null in the first pass, which forms them
    uint32_t *key, *pos;
    uint32_t *hist, *total;
    uint32_t tiles;
    int shift, bits;
    uint32_t *seen;           // a bit for every token of the table that occurs (the first pass sets them; may be null)
    ZeroTable z;              // and this launch's share of the zero rows, for the CTAs after the sort's
    int64_t zero0, zero1, rows_per_cta;
};

constexpr int kSeenWords = 4096;

// A CTA's part of the zero rows of a launch; `index` counts those CTAs.
__device__ __forceinline__ void zero_share(const TileSortArgs &a, unsigned index)
{
    const int64_t row0 = a.zero0 + index * a.rows_per_cta, row1 = min(a.zero1, row0 + a.rows_per_cta);
    for (int64_t v = row0 + (threadIdx.x >> 5); v < row1; v += blockDim.x >> 5)
        if (!(a.seen[v >> 5] >> (v & 31) & 1u)) zero_row(a.z.dw + v * a.e.table_stride * a.z.elem, a.e.dim * a.z.elem);
}

template <int ITEMS>
__device__ __forceinline__ void load_tile(const TileSortArgs &a, uint2 (&item)[ITEMS], uint32_t (&digit)[ITEMS], bool report)
{
    const uint32_t slot0 = blockIdx.x * kTile1 + (threadIdx.x >> 5) * 32 * ITEMS + (threadIdx.x & 31);
    const uint32_t n = static_cast<uint32_t>(a.e.n);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t t = slot0 + 32 * i;
        item[i] = make_uint2(0xffffffffu, t);
        if (t < n) item[i] = a.key_in ? make_uint2(a.key_in[t], a.pos_in[t]) : make_uint2(key_at(a.e, t, report), t);
        digit[i] = (item[i].x >> a.shift) & ((1u << a.bits) - 1);
    }
}

__global__ void __launch_bounds__(kSortThreads) hist_kernel(const TileSortArgs a)
{
    __shared__ uint32_t count[kDigits], here[kSeenWords];
    pdl_trigger();
    const bool mark = a.seen && !a.key_in, gather = mark && a.e.vocab <= 32 * kSeenWords;
    const int words = static_cast<int>((min(a.e.vocab, int64_t{32} * kSeenWords) + 31) / 32);
    if (threadIdx.x < kDigits) count[threadIdx.x] = 0;
    if (gather)
        for (int i = threadIdx.x; i < words; i += kSortThreads) here[i] = 0;
    pdl_wait();
    if (blockIdx.x >= a.tiles) return zero_share(a, blockIdx.x - a.tiles);
    __syncthreads();
    uint2 item[kTileItems];
    uint32_t digit[kTileItems];
    load_tile(a, item, digit, true);
    // Tokens that occur: each CTA's are gathered in shared memory first, so that a frequent token is one request a CTA
    // and a warp looks at 32 words of the table's bits at a time (a table of up to 32 kSeenWords tokens).
    if (mark)
#pragma unroll
        for (int i = 0; i < kTileItems; ++i)
            if (item[i].x < a.e.vocab) atomicOr(&(gather ? here : a.seen)[item[i].x >> 5], 1u << (item[i].x & 31));
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const uint32_t peers = __match_any_sync(0xffffffffu, digit[i]);
        if ((threadIdx.x & 31) == __ffs(peers) - 1) atomicAdd(&count[digit[i]], static_cast<uint32_t>(__popc(peers)));
    }
    __syncthreads();
    if (threadIdx.x < (1u << a.bits)) a.hist[static_cast<size_t>(threadIdx.x) * a.tiles + blockIdx.x] = count[threadIdx.x];
    if (gather)
        for (int i = threadIdx.x; i < words; i += kSortThreads)
            if (here[i] & ~*static_cast<volatile uint32_t *>(a.seen + i)) atomicOr(a.seen + i, here[i]);
}

// One CTA per digit: its counts become exclusive sums over the tiles, total[d] their sum.
__global__ void __launch_bounds__(kSortThreads) scan_kernel(const TileSortArgs a)
{
    __shared__ uint32_t warp_sums[kSortWarps];
    pdl_trigger();
    pdl_wait();
    if (blockIdx.x >= 1u << a.bits) return zero_share(a, blockIdx.x - (1u << a.bits));
    const uint32_t tiles = a.tiles;
    uint32_t *row = a.hist + static_cast<size_t>(blockIdx.x) * tiles, carry = 0;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    for (uint32_t i0 = 0; i0 < tiles; i0 += kSortThreads) {
        const uint32_t i = i0 + threadIdx.x, v = i < tiles ? row[i] : 0;
        uint32_t sum = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += up;
        }
        if (lane == 31) warp_sums[w] = sum;
        __syncthreads();
        uint32_t before = carry, all = 0;
#pragma unroll
        for (int k = 0; k < kSortWarps; ++k) {
            before += k < w ? warp_sums[k] : 0;
            all += warp_sums[k];
        }
        if (i < tiles) row[i] = before + sum - v;
        carry += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.total[blockIdx.x] = carry;
}

__global__ void __launch_bounds__(kSortThreads) scatter_kernel(const TileSortArgs a)
{
    __shared__ uint32_t hist[kSortWarps][kDigits], total[kDigits], base[kDigits], warp_sums[kDigits / 32];
    pdl_trigger();
    pdl_wait();
    if (blockIdx.x >= a.tiles) return zero_share(a, blockIdx.x - a.tiles);
    uint2 item[kTileItems];
    uint32_t digit[kTileItems], rank[kTileItems];
    load_tile(a, item, digit, false);
    const int digits = 1 << a.bits;
    rank_digits(digit, rank, hist, total, digits);
    const bool mine = threadIdx.x < digits;
    scan_digits(mine ? a.total[threadIdx.x] : 0, mine ? a.hist[static_cast<size_t>(threadIdx.x) * a.tiles + blockIdx.x] : 0, base,
                warp_sums);
    const uint32_t n = static_cast<uint32_t>(a.e.n);
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const uint32_t at = base[digit[i]] + hist[threadIdx.x >> 5][digit[i]] + rank[i];
        if (at < n) {  // the last tile's empty slots come last
            a.key[at] = item[i].x;
            a.pos[at] = item[i].y;
        }
    }
}

struct SumArgs {
    EmbedArgs e;
    const uint32_t *key, *pos;
    float *partial;       // chunk c's head at 2 c * pad, its tail at (2 c + 1) * pad
    int64_t pad;          // columns of a partial sum, a multiple of 8
    int64_t chunk;        // entries of the list per chunk
    int accumulate;
};

template <class W, int VEC>
__device__ __forceinline__ void store_sums(W *p, const float (&sum)[VEC], float scale, int accumulate)
{
    Pack<W, VEC> x;
    if (accumulate) load_pack<W, VEC>(p, x);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float s = __fmul_rn(sum[i], scale);
        x.y[i] = from_f32<W>(accumulate ? __fadd_rn(to_f32(x.y[i]), s) : s);
    }
    store_pack<W, VEC>(p, x);
}

constexpr int kSumThreads = 256;
constexpr int kSumRows = 512;   // entries of the list that a CTA holds in shared memory at a time
constexpr int kSumGroup = 4;    // rows of one group of asynchronous copies
constexpr int kSumGroups = 4;   // groups in flight and in use

// Bytes of the ring of rows in shared memory.
inline size_t sum_smem(int vec, int threads) { return vec > 1 ? size_t{kSumGroup} * kSumGroups * threads * 16 : 0; }

// A thread owns VEC columns of its chunk's rows.  Rows come through a ring in shared memory filled by asynchronous
// copies, each thread copying and reading its own 16 bytes (no barrier between rows), so that as many rows as the ring
// holds are in flight while the sum goes on; single elements (VEC = 1) are loaded a group at a time.
template <class Y, class W, int VEC>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const SumArgs a, const Y *dy, W *dw)
{
    __shared__ uint32_t keys[kSumRows];
    __shared__ int64_t rows[kSumRows];
    extern __shared__ uint4 ring[];
    pdl_trigger();
    pdl_wait();
    const int64_t chunk = blockIdx.x, begin = chunk * a.chunk, end = min(a.e.n, begin + a.chunk);
    const int64_t j = (static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x) * VEC;
    const uint32_t none = static_cast<uint32_t>(a.e.vocab);
    const bool in = j < a.e.dim;
    const uint32_t first = a.key[begin], before = begin > 0 ? a.key[begin - 1] : none;
    const uint32_t tail = a.key[end - 1], after = end < a.e.n ? a.key[end] : none;
    if (first == none) return;  // nothing but tokens without a gradient from here on
    const bool head_in = before == first, goes_on = tail != none && tail == after;  // runs that cross the chunk's borders
    float *part = a.partial + 2 * chunk * a.pad + j;
    float sum[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) sum[k] = 0.0f;
    uint32_t cur = first;
    bool from_head = head_in;
    // The end of the run of `cur`, or of the chunk within one.
    auto flush = [&](bool crosses) {
        if (!in) return;
        if (from_head || crosses) {
            float *p = part + (from_head ? 0 : a.pad);
#pragma unroll
            for (int k = 0; k < VEC; ++k) p[k] = sum[k];
        } else {
            store_sums<W, VEC>(dw + cur * a.e.table_stride + j, sum, a.e.scale, a.accumulate);
        }
    };
    for (int64_t b = begin; b < end; b += kSumRows) {
        const int n = static_cast<int>(min(end - b, static_cast<int64_t>(kSumRows)));
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            keys[i] = a.key[b + i];
            rows[i] = row_at(a.e, a.pos[b + i]);
        }
        __syncthreads();
        auto wanted = [&](int i) { return in && i < n && keys[i] != none; };
        auto fetch = [&](int i0) {  // rows i0 .. i0 + kSumGroup - 1 into their places in the ring
            if constexpr (VEC > 1) {
#pragma unroll
                for (int u = 0; u < kSumGroup; ++u)
                    if (wanted(i0 + u)) cp_async16(&ring[((i0 + u) % (kSumGroup * kSumGroups)) * blockDim.x + threadIdx.x], dy + rows[i0 + u] + j);
                cp_async_commit();
            }
        };
#pragma unroll
        for (int g = 0; g < kSumGroups - 1; ++g) fetch(g * kSumGroup);
        for (int i = 0; i < n; i += kSumGroup) {
            Pack<Y, VEC> x[kSumGroup];
            if constexpr (VEC > 1) {
                fetch(i + (kSumGroups - 1) * kSumGroup);
                cp_async_wait<kSumGroups - 1>();
#pragma unroll
                for (int u = 0; u < kSumGroup; ++u)
                    *reinterpret_cast<uint4 *>(&x[u]) = ring[((i + u) % (kSumGroup * kSumGroups)) * blockDim.x + threadIdx.x];
            } else {
#pragma unroll
                for (int u = 0; u < kSumGroup; ++u)
                    if (wanted(i + u)) x[u].y[0] = dy[rows[i + u] + j];
            }
#pragma unroll
            for (int u = 0; u < kSumGroup; ++u) {
                if (i + u >= n) break;
                const uint32_t k = keys[i + u];
                if (k != cur) {
                    flush(false);
                    cur = k;
                    from_head = false;
#pragma unroll
                    for (int v = 0; v < VEC; ++v) sum[v] = 0.0f;
                    if (k == none) {
                        cp_async_wait_all();
                        return;
                    }
                }
#pragma unroll
                for (int v = 0; v < VEC; ++v) sum[v] = __fadd_rn(sum[v], to_f32(x[u].y[v]));
            }
        }
    }
    flush(goes_on);
}

constexpr int kCombineThreads = 256, kCombineSplit = 4;

// The rows of the tokens whose runs cross chunks.  CTA (c, y) takes the run that starts in chunk c and goes on in
// the next, if there is one -- the tail of c and the heads of the chunks after it, as far as the run goes -- and
// every kCombineSplit-th piece of its columns.  The more chunks a run has, the more groups of threads take them in
// turn; the groups' sums are added in order.
template <class W>
__global__ void __launch_bounds__(kCombineThreads) combine_kernel(const SumArgs a, W *dw)
{
    __shared__ float4 red[kCombineThreads];
    pdl_wait();
    const int64_t c = blockIdx.x, begin = c * a.chunk, next = begin + a.chunk;  // c is not the last chunk
    const uint32_t none = static_cast<uint32_t>(a.e.vocab), v = a.key[next], tail = a.key[next - 1], first = a.key[begin],
                   before = begin > 0 ? a.key[begin - 1] : none;
    if (v == none || tail != v || (first == v && before == v)) return;
    int64_t last = c + 1;  // the chunks whose first entry is v: c + 1 .. last
    for (int64_t k = c + 2;; k += 32) {
        const int64_t at = (k + (threadIdx.x & 31)) * a.chunk;
        const uint32_t same = __ballot_sync(0xffffffffu, at < a.e.n && a.key[at] == v);
        const int run = same == 0xffffffffu ? 32 : __ffs(~same) - 1;
        last += run;
        if (run < 32) break;
    }
    const int64_t parts = last - c;
    const int groups = parts > 32 ? 8 : parts > 16 ? 4 : parts > 8 ? 2 : 1, width = kCombineThreads / groups;
    const int group = threadIdx.x / width, lane = threadIdx.x % width;
    for (int64_t j0 = static_cast<int64_t>(blockIdx.y) * width * 4; j0 < a.e.dim; j0 += static_cast<int64_t>(kCombineSplit) * width * 4) {
        const int64_t j = j0 + lane * 4;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (j < a.e.dim) {
            if (group == 0) sum = *reinterpret_cast<const float4 *>(a.partial + (2 * c + 1) * a.pad + j);
#pragma unroll 8
            for (int64_t k = c + 1 + group; k <= last; k += groups) {
                const float4 x = *reinterpret_cast<const float4 *>(a.partial + 2 * k * a.pad + j);
                sum = make_float4(__fadd_rn(sum.x, x.x), __fadd_rn(sum.y, x.y), __fadd_rn(sum.z, x.z), __fadd_rn(sum.w, x.w));
            }
        }
        if (groups > 1) {
            __syncthreads();
            red[threadIdx.x] = sum;
            __syncthreads();
        }
        if (group == 0) {
            for (int g = 1; g < groups; ++g) {
                const float4 x = red[g * width + lane];
                sum = make_float4(__fadd_rn(sum.x, x.x), __fadd_rn(sum.y, x.y), __fadd_rn(sum.z, x.z), __fadd_rn(sum.w, x.w));
            }
            const float s[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (j + i < a.e.dim) store_sums<W, 1>(dw + v * a.e.table_stride + j + i, {s[i]}, a.e.scale, a.accumulate);
        }
    }
}

}  // namespace ea

using namespace ea;

struct ea_embed {
    DeviceOf dev;
    cudaStream_t stream = nullptr;
    ea_embed_config cfg{};
    uint32_t *status = nullptr;
    uint32_t *key[2] = {}, *pos[2] = {};  // the sorted list; the second pair, hist, total and seen: longer sorts only
    uint32_t *hist = nullptr, *total = nullptr, *seen = nullptr;
    float *partial = nullptr;
};

namespace {

int validate(const ea_embed_config *cfg)
{
    if (!cfg) return lm_fail(EA_E_INVAL, "config is NULL");
    if (cfg->vocab < 1 || cfg->vocab > 0x7ffffffeLL) return lm_fail(EA_E_INVAL, "vocab must be in [1, 2^31 - 2]");
    if (cfg->dim < 1 || cfg->dim > (1 << 20)) return lm_fail(EA_E_INVAL, "dim must be in [1, 2^20]");
    if (cfg->max_tokens < 0 || cfg->max_tokens > (1 << 30)) return lm_fail(EA_E_INVAL, "max_tokens must be in [0, 2^30]");
    if (cfg->padding < -1 || cfg->padding >= cfg->vocab) return lm_fail(EA_E_INVAL, "padding must be a token or -1");
    if (!std::isfinite(cfg->scale)) return lm_fail(EA_E_INVAL, "scale must be finite");
    return EA_OK;
}

constexpr int kMaxVec = 8;
constexpr int kMinChunk = 8;

int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }
int64_t over(int64_t x, int64_t a) { return (x + a - 1) / a; }

// How sum_kernel's CTAs share the columns: `slabs` of them side by side, of `threads` threads.
struct SumShape {
    int64_t slabs;
    int threads;
    SumShape(int64_t dim, int vec)
    {
        const int64_t packs = over(dim, vec);
        slabs = over(packs, kSumThreads);
        threads = static_cast<int>(up(over(packs, slabs), 32));
    }
};

// Chunks that the sorted list is cut into at most.  The cut decides which binary32 sums are formed before they are
// joined, so it goes by the width alone, whatever the types, the rows' alignment and the device: 1,024 threads on each of
// 152 SMs where rows are read in packs of kMaxVec, slabs counted.  Binary32 rows, which fill as many threads with half as
// many chunks: 260,096 x 768 186 us (with half as many chunks 203), half of them padding 134 (123); 16,384 x 1600 90.6 (90.2).
constexpr int kCutSms = 152;
int64_t most_chunks(int64_t dim)
{
    const SumShape shape(dim, kMaxVec);
    return std::max<int64_t>(1, kCutSms * (1024 / shape.threads) / shape.slabs);
}

// Entries per chunk, no fewer than kMinChunk (a chunk may write two partial sums, as many bytes as 4 rows in 16 bits).
// With 4, 8 and 16: 384 tokens x 768 in 32 bits 12.4, 12.4 and 15.1 us; 2,000 x 1600 in 16 bits 24.9, 21.0 and 22.6.
int64_t chunk_length(int64_t n, int64_t dim) { return std::max<int64_t>(kMinChunk, over(n, most_chunks(dim))); }

struct EmbedLayout {
    size_t status, list, hist, total_, seen, partial;
    int lists;
    size_t total() const { return status + 2 * lists * list + hist + total_ + seen + partial; }
};

EmbedLayout embed_layout(const ea_embed_config &cfg)
{
    const int64_t n = cfg.max_tokens;
    EmbedLayout l{};
    l.status = 256;
    l.list = up(n * 4, 256);
    l.lists = n > kClusterTokens ? 2 : 1;
    if (n > kClusterTokens) {
        l.hist = up(over(n, kTile1) * kDigits * 4, 256);
        l.total_ = kDigits * 4;
        l.seen = up(over(cfg.vocab, 32) * 4, 256);
    }
    l.partial = 2 * std::min(over(n, kMinChunk), most_chunks(cfg.dim)) * up(cfg.dim, kMaxVec) * 4;  // all that chunk_length allows
    return l;
}

// The quotient by d >= 2 of a number below 2^30 is its product with magic, shifted by 32 + shift (see batch_row).
void set_divisor(uint32_t d, uint32_t &magic, int &shift)
{
    int s = 0;
    while ((int64_t{1} << s) < d) ++s;
    magic = static_cast<uint32_t>((uint64_t{1} << (31 + s)) / d + 1);
    shift = s - 1;
}

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
    a = EmbedArgs{};
    a.n = c->outer * c->inner;
    a.token_outer = c->token_outer;
    a.token_inner = c->token_inner;
    a.row_outer = c->row_outer;
    a.row_inner = c->row_inner;
    if (c->inner == 1) {  // a column of the batch is a row of it
        a.token_inner = c->token_outer;
        a.row_inner = c->row_outer;
    } else if (c->outer > 1 && (c->token_outer != c->inner * c->token_inner || c->row_outer != c->inner * c->row_inner)) {
        a.inner = static_cast<uint32_t>(c->inner);
        set_divisor(a.inner, a.magic, a.shift);
    }
    a.table_stride = c->table_stride;
    a.vocab = h->cfg.vocab;
    a.dim = h->cfg.dim;
    a.padding = h->cfg.padding;
    a.scale = h->cfg.scale;
    a.token64 = c->token_type == EA_T_I64;
    a.tokens = tokens;
    a.status = h->status;
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

// Whether every row of a tensor starts on a 16-byte boundary and is whole vectors of it.
bool rows_aligned(const void *p, int32_t type, int64_t dim, int64_t outer, int64_t inner)
{
    const int64_t vec = 16 / static_cast<int64_t>(type_bytes(type));
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && dim % vec == 0 && outer % vec == 0 && inner % vec == 0;
}

// f(std::integral_constant<int, ITEMS>) for the keys per thread that n tokens take in a cluster of `ctas`.
template <class F>
void with_items(int64_t n, int ctas, F f)
{
    const int64_t items = over(n, int64_t{kSortThreads} * ctas);
    if (items <= 1) f(std::integral_constant<int, 1>());
    else if (items <= 2) f(std::integral_constant<int, 2>());
    else if (items <= 4) f(std::integral_constant<int, 4>());
    else if (items <= 8) f(std::integral_constant<int, 8>());
    else f(std::integral_constant<int, kMaxItems>());
}

int allow_sort_smem()
{
    auto allow = [](auto *kernel, size_t bytes) {
        return lm_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)), "shared memory");
    };
    int r = EA_OK;
    for (int32_t yt : {EA_T_F32, EA_T_BF16, EA_T_F16})
        for (int32_t wt : {EA_T_F32, EA_T_BF16, EA_T_F16})
            with_type(yt, [&](auto *y) {
                with_type(wt, [&](auto *w) {
                    using Y = std::remove_reference_t<decltype(*y)>;
                    using W = std::remove_reference_t<decltype(*w)>;
                    if (r == EA_OK) r = allow(sum_kernel<Y, W, 16 / sizeof(Y)>, sum_smem(2, kSumThreads));
                });
            });
    if (r == EA_OK) r = allow(order_kernel<4>, kSortSmem<4>);
    if (r == EA_OK) r = allow(order_kernel<8>, kSortSmem<8>);
    if (r == EA_OK) r = allow(order_kernel<kMaxItems>, kSortSmem<kMaxItems>);
    return r;
}

// The sorted list of the tokens into h.key[0], h.pos[0]; with `zero`, the rows of dw whose token does not occur.
int order_tokens(ea_embed &h, const EmbedArgs &a, const ZeroTable &z, bool zero)
{
    int key_bits = 1;
    while ((a.vocab >> key_bits) != 0) ++key_bits;  // keys are 0 .. vocab
    const int passes = static_cast<int>(over(key_bits, 8)), bits = static_cast<int>(over(key_bits, passes));
    cudaError_t e = cudaSuccess;
    if (a.n <= kClusterTokens) {
        const int ctas = a.n <= kOneCtaTokens ? 1 : kCluster;
        const int64_t rows = over(a.vocab, h.dev.sms * kZeroCtasPerSm), zero_ctas = zero ? up(over(a.vocab, rows), ctas) : 0;
        with_items(a.n, ctas, [&](auto items) {
            constexpr int kItems = decltype(items)::value;
            const SortArgs s{a, h.key[0], h.pos[0], passes, bits};
            e = launch_lm(order_kernel<kItems>, dim3(static_cast<unsigned>(ctas + zero_ctas)), kSortThreads, kSortSmem<kItems>, h.stream,
                          false, ctas, s, z, rows);
        });
        return lm_cuda(e, "launch");
    }
    TileSortArgs s{};
    s.e = a;
    s.hist = h.hist;
    s.total = h.total;
    s.tiles = static_cast<uint32_t>(over(a.n, kTile1));
    s.bits = bits;
    s.seen = zero ? h.seen : nullptr;
    s.z = z;
    if (zero) e = cudaMemsetAsync(h.seen, 0, over(a.vocab, 32) * 4, h.stream);
    const int launches = 3 * passes - 1;  // that write zero rows: all but the first
    int done = -1;
    auto launch = [&](auto *kernel, unsigned grid) {
        s.zero0 = s.zero1 = 0;
        s.rows_per_cta = 1;
        unsigned zero_ctas = 0;
        if (zero && done >= 0) {
            s.zero0 = a.vocab * done / launches;
            s.zero1 = a.vocab * (done + 1) / launches;
            s.rows_per_cta = std::max<int64_t>(1, over(s.zero1 - s.zero0, h.dev.sms * 2));
            zero_ctas = static_cast<unsigned>(over(s.zero1 - s.zero0, s.rows_per_cta));
        }
        if (e == cudaSuccess) e = launch_lm(kernel, dim3(grid + zero_ctas), kSortThreads, 0, h.stream, done >= 0, 1, s);
        ++done;
    };
    for (int pass = 0; pass < passes; ++pass) {
        const int to = (passes - 1 - pass) & 1;  // the last pass writes the first pair
        s.key_in = pass ? h.key[to ^ 1] : nullptr;
        s.pos_in = pass ? h.pos[to ^ 1] : nullptr;
        s.key = h.key[to];
        s.pos = h.pos[to];
        s.shift = pass * bits;
        launch(hist_kernel, s.tiles);
        launch(scan_kernel, 1u << bits);
        launch(scatter_kernel, s.tiles);
    }
    return lm_cuda(e, "launch");
}

}  // namespace

extern "C" {

int ea_embed_workspace_bytes(const ea_embed_config *cfg, size_t *bytes)
{
    if (!bytes) return lm_fail(EA_E_INVAL, "bytes is NULL");
    const int r = validate(cfg);
    if (r != EA_OK) return r;
    *bytes = embed_layout(*cfg).total();
    return EA_OK;
}

int ea_embed_init(const ea_embed_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_embed **out)
{
    if (!out) return lm_fail(EA_E_INVAL, "out is NULL");
    *out = nullptr;
    int r = validate(cfg);
    if (r != EA_OK) return r;
    if ((r = check_workspace(workspace, workspace_bytes, embed_layout(*cfg).total())) != EA_OK) return r;
    ea_embed *h = new (std::nothrow) ea_embed;
    if (!h) return lm_fail(EA_E_INVAL, "out of host memory");
    h->cfg = *cfg;
    h->stream = static_cast<cudaStream_t>(stream);
    const EmbedLayout l = embed_layout(*cfg);
    unsigned char *p = static_cast<unsigned char *>(workspace);
    auto take = [&p](size_t bytes) {
        unsigned char *q = p;
        p += bytes;
        return q;
    };
    h->status = reinterpret_cast<uint32_t *>(take(l.status));
    for (int i = 0; i < l.lists; ++i) {
        h->key[i] = reinterpret_cast<uint32_t *>(take(l.list));
        h->pos[i] = reinterpret_cast<uint32_t *>(take(l.list));
    }
    h->hist = reinterpret_cast<uint32_t *>(take(l.hist));
    h->total = reinterpret_cast<uint32_t *>(take(l.total_));
    h->seen = reinterpret_cast<uint32_t *>(take(l.seen));
    h->partial = reinterpret_cast<float *>(take(l.partial));
    r = h->dev.query();
    h->dev.sms = std::min(h->dev.sms, kMaxSms);
    if (r == EA_OK) r = allow_sort_smem();
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
    const int vec = rows_aligned(y, c->row_type, a.dim, c->outer > 1 ? c->row_outer : 0, c->inner > 1 ? c->row_inner : 0) &&
                            rows_aligned(w, c->table_type, a.dim, a.table_stride, 0)
                        ? 16 / static_cast<int>(type_bytes(c->table_type)) : 1;
    const uint32_t packs = static_cast<uint32_t>(a.dim / vec);
    with_type(c->table_type, [&](auto *wt) {
        using W = std::remove_reference_t<decltype(*wt)>;
        with_type(c->row_type, [&](auto *yt) {
            using Y = std::remove_reference_t<decltype(*yt)>;
            constexpr int kVec = 16 / sizeof(W);
            const W *from = static_cast<const W *>(w);
            Y *to = static_cast<Y *>(y);
            if (packs >= kWideRow) {
                LookupWideArgs l{};
                l.e = a;
                l.packs = packs;
                l.pieces = static_cast<uint32_t>(over(packs, 32 * kWideUnroll));
                l.piece = static_cast<uint32_t>(up(over(packs, l.pieces), 32));
                l.total = a.n * l.pieces;
                const int64_t warps = kLookupThreads / 32, ctas = std::min<int64_t>(over(l.total, warps), h->dev.sms * kLookupCtasPerSm);
                l.turn_rows = static_cast<uint32_t>(ctas * warps / l.pieces);
                l.turn_pieces = static_cast<uint32_t>(ctas * warps % l.pieces);
                auto kernel = vec > 1 ? lookup_wide_kernel<W, Y, kVec> : lookup_wide_kernel<W, Y, 1>;
                kernel<<<static_cast<unsigned>(ctas), kLookupThreads, 0, h->stream>>>(l, from, to);
            } else {
                LookupArgs l{};
                l.e = a;
                l.packs = packs;
                l.total = a.n * packs;
                if (packs > 1) set_divisor(packs, l.magic, l.shift);
                const int64_t span = kLookupThreads * kLookupUnroll;
                const int64_t ctas = std::min<int64_t>(over(l.total, span), h->dev.sms * kLookupCtasPerSm);
                l.turn_rows = static_cast<uint32_t>(ctas * span / packs);
                l.turn_packs = static_cast<uint32_t>(ctas * span % packs);
                auto kernel = vec > 1 ? lookup_narrow_kernel<W, Y, kVec> : lookup_narrow_kernel<W, Y, 1>;
                kernel<<<static_cast<unsigned>(ctas), kLookupThreads, 0, h->stream>>>(l, from, to);
            }
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
    if (a.n == 0 && accumulate) return EA_OK;
    const int wb = static_cast<int>(type_bytes(c->table_type));
    const ZeroTable z{static_cast<unsigned char *>(dw), wb};
    const int ordered = order_tokens(*h, a, z, !accumulate);
    if (ordered != EA_OK || a.n == 0) return ordered;
    cudaError_t e = cudaSuccess;
    const int vec = rows_aligned(dy, c->row_type, a.dim, c->outer > 1 ? c->row_outer : 0, c->inner > 1 ? c->row_inner : 0) &&
                            rows_aligned(dw, c->table_type, a.dim, a.table_stride, 0)
                        ? 16 / static_cast<int>(type_bytes(c->row_type)) : 1;
    const SumShape shape(a.dim, vec);
    const SumArgs s{a, h->key[0], h->pos[0], h->partial, up(a.dim, kMaxVec), chunk_length(a.n, a.dim), accumulate};
    const unsigned chunks = static_cast<unsigned>(over(a.n, s.chunk));
    with_type(c->row_type, [&](auto *yt) {
        using Y = std::remove_reference_t<decltype(*yt)>;
        with_type(c->table_type, [&](auto *wt) {
            using W = std::remove_reference_t<decltype(*wt)>;
            const dim3 grid(chunks, static_cast<unsigned>(shape.slabs));
            auto kernel = vec > 1 ? sum_kernel<Y, W, 16 / sizeof(Y)> : sum_kernel<Y, W, 1>;
            e = launch_lm(kernel, grid, shape.threads, sum_smem(vec, shape.threads), h->stream, true, 1, s, static_cast<const Y *>(dy),
                          static_cast<W *>(dw));
            if (e == cudaSuccess && chunks > 1)
                e = launch_lm(combine_kernel<W>, dim3(chunks - 1, kCombineSplit), kCombineThreads, 0, h->stream, true, 1, s,
                              static_cast<W *>(dw));
        });
    });
    return lm_cuda(e, "launch");
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
