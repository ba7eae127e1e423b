// Lookup of table rows by tokens and its gradient (tad_embed_forward, tad_embed_backward).
//
//     y_t = factor E_{tok_t},        dE_v = factor sum_{t : tok_t = v} dy_t
//
// The gradient is the gather form of the derivative for an index that is data: Gamma(v) = { t : tok_t = v } comes from sorting
// the positions by token instead of from an inverse index map.  A stable radix sort keeps each row's positions in ascending
// order, so the sums have a fixed order without atomics.
//
// Both directions move bytes and are bound by memory: the gradient reads dy once (rows in sorted order, whole rows at a time)
// and writes the table's gradient once, zeros included.
#include <cooperative_groups.h>

#include <atomic>
#include <type_traits>

#include "rows.cuh"

namespace {

using namespace tadr;

// a token as the key it is sorted by: n_table for everything outside the table
struct Tokens {
    const void *p;
    int bits;
    unsigned n_table;
    __device__ __forceinline__ unsigned key(int64_t t) const
    {
        const long long k = bits == 32 ? (long long)static_cast<const int *>(p)[t] : static_cast<const long long *>(p)[t];
        return k >= 0 && k < (long long)n_table ? (unsigned)k : n_table;
    }
};

// ---- forward ----

constexpr int NT = 256, ROWS = 4;

// ROWS rows of V elements a thread; 2^log threads stand beside each other in a row
template <class S, class T, int V>
__global__ void __launch_bounds__(NT)
tad_embed_forward_kernel(const Tokens tok, int64_t n, const S *__restrict__ table, int64_t ts, int width, float factor, T *__restrict__ y,
                         int64_t ys, int log, unsigned chunks)
{
    tad_wait_previous();
    const unsigned group = blockIdx.x / chunks, chunk = blockIdx.x - group * chunks;
    const int step = NT >> log;
    const int64_t t0 = (int64_t)group * (ROWS * step) + (threadIdx.x >> log);
    const int64_t c = ((int64_t)(chunk << log) + (threadIdx.x & ((1 << log) - 1))) * V;
    if (c >= width) return;
    unsigned key[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) key[i] = t0 + i * step < n ? tok.key(t0 + i * step) : tok.n_table;
    Piece<S, V> p[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        p[i].zero();
        if (key[i] < tok.n_table) p[i].load(table + (int64_t)key[i] * ts + c);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (t0 + i * step >= n) continue;
        float v[V];
        p[i].get(v);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = key[i] < tok.n_table ? v[j] * factor : 0.f;      // (zeros even where the factor is not finite)
        Piece<T, V> o;
        o.set(v);
        o.store(y + (t0 + i * step) * ys + c);
    }
}

// ---- the sort ----

// One cluster of blocks sorts (key, position) by digits of at most nine bits, least digit first.  A warp owns a run of consecutive
// elements and counts its digits in shared memory (lanes with equal digits find each other by a vote, one of them adds); the
// counts of a digit are prefixed over the warps of a block, the blocks of the cluster (read from each other's shared memory) and the
// digits; then the warp walks its run again and every element knows its place.  One launch for the whole sort, a cluster
// barrier where a grid of independent blocks would need a launch: the arrays stay in L2.
constexpr int SORT_NT = 1024, SORT_WARPS = SORT_NT / 32, DIGITS = 512;
constexpr size_t SORT_SMEM = SORT_WARPS * DIGITS * 4;

__global__ void __launch_bounds__(SORT_NT)
tad_embed_sort_kernel(const Tokens tok, unsigned n, unsigned run, int passes, int bits, unsigned *k0, unsigned *p0, unsigned *k1, unsigned *p1)
{
    namespace cg = cooperative_groups;
    extern __shared__ unsigned counts[];                       // of a warp: counts[warp * DIGITS + digit]
    __shared__ unsigned total[DIGITS], sums[32];
    cg::cluster_group cluster = cg::this_cluster();
    const unsigned rank = cluster.block_rank(), blocks = cluster.num_blocks();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int digits = 1 << bits;
    const unsigned long long first = (unsigned long long)(rank * SORT_WARPS + warp) * run;
    const unsigned beg = (unsigned)min((unsigned long long)n, first), end = (unsigned)min((unsigned long long)n, first + run);
    unsigned *mine = counts + warp * DIGITS;
    tad_wait_previous();
    for (int pass = 0; pass < passes; ++pass) {
        const unsigned *ki = pass & 1 ? k0 : k1, *pi = pass & 1 ? p0 : p1;
        unsigned *ko = pass & 1 ? k1 : k0, *po = pass & 1 ? p1 : p0;
        const int shift = pass * bits;
        // (written by other blocks of the cluster in the pass before: not from the first-level cache)
        auto key_at = [&](unsigned t) { return pass == 0 ? tok.key(t) : __ldcg(ki + t); };
        for (int d = lane; d < digits; d += 32) mine[d] = 0;
        __syncwarp();
        for (unsigned t0 = beg; t0 < end; t0 += 32) {
            const unsigned t = t0 + lane;
            const bool live = t < end;
            const unsigned d = live ? (key_at(t) >> shift) & (digits - 1) : 0xffffffffu;
            const unsigned same = __match_any_sync(0xffffffffu, d);
            if (live && (same & ((1u << lane) - 1)) == 0) mine[d] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        const int d = threadIdx.x;
        if (d < digits) {
            unsigned a = 0;
            for (int w = 0; w < SORT_WARPS; ++w) { const unsigned c = counts[w * DIGITS + d]; counts[w * DIGITS + d] = a; a += c; }
            total[d] = a;
        }
        cluster.sync();
        unsigned before = 0, all = 0;
        if (d < digits)
            for (unsigned b = 0; b < blocks; ++b) {
                const unsigned c = cluster.map_shared_rank(total, b)[d];
                if (b < rank) before += c;
                all += c;
            }
        // exclusive prefix over the digits
        unsigned up = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const unsigned x = __shfl_up_sync(0xffffffffu, up, o); if (lane >= o) up += x; }
        if (lane == 31) sums[warp] = up;
        __syncthreads();
        unsigned base = lane < warp ? sums[lane] : 0;
#pragma unroll
        for (int o = 16; o; o >>= 1) base += __shfl_xor_sync(0xffffffffu, base, o);
        base += up - all + before;
        if (d < digits)
            for (int w = 0; w < SORT_WARPS; ++w) counts[w * DIGITS + d] += base;
        __syncthreads();
        for (unsigned t0 = beg; t0 < end; t0 += 32) {
            const unsigned t = t0 + lane;
            const bool live = t < end;
            const unsigned key = live ? key_at(t) : 0;
            const unsigned e = live ? (key >> shift) & (digits - 1) : 0xffffffffu;
            const unsigned same = __match_any_sync(0xffffffffu, e);
            const unsigned lower = __popc(same & ((1u << lane) - 1));
            if (live) {
                const unsigned to = mine[e] + lower;
                ko[to] = key;
                po[to] = pass == 0 ? t : __ldcg(pi + t);
            }
            __syncwarp();
            if (live && lower == 0) mine[e] += __popc(same);
            __syncwarp();
        }
        cluster.sync();
    }
}

// ---- the sums ----

// Row ends 0 .. n_table - 1 and sorted tokens are merged into one list (the tokens of a row before its end) that is cut into segments of
// equal length, so neither a table much longer than the batch nor a token that is half of the batch leaves warps idle.  A warp
// owns a segment in 256 columns: a token adds its row of dy to the registers, a row end writes them.  A row that
// begins in one segment and ends in another leaves a partial sum in each: `tail` of the segments that it does not end in, `head` of
// the one it ends in; tad_embed_join_kernel adds them up in order.
constexpr int SLICE = 256, AHEAD = 4;

struct Cut {
    unsigned first_row;      // the row that is open at the segment's begin
    unsigned state;          // OPEN: tokens of it lie in segments before;  ENDS: it ends in this segment
};
constexpr unsigned OPEN = 1, ENDS = 2;

struct Sums {
    const unsigned *keys, *at;
    const void *dy;
    int64_t dys;
    void *dtable;
    int64_t ds;
    int type, accumulate;
    unsigned n, n_table, segments, slices;
    int64_t each;            // length of a segment
    int width;
    float factor;
    float *head, *tail;
    Cut *cuts;
};

// tokens among the first d entries of the merged list: the first i with keys[i] > d - 1 - i, by the lanes of a warp at once
__device__ __forceinline__ unsigned tokens_before(const unsigned *__restrict__ keys, unsigned n, unsigned n_table, int64_t d)
{
    const int lane = threadIdx.x & 31;
    int64_t lo = d > n_table ? d - n_table : 0, hi = d < (int64_t)n ? d : (int64_t)n;          // the answer lies in [lo, hi]
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32, i = lo + lane * step;
        const bool before = i < hi && (int64_t)keys[i] <= d - 1 - i;
        const int k = __popc(__ballot_sync(0xffffffffu, before));                             // (true for the first k lanes)
        if (k == 0) return (unsigned)lo;
        const int64_t low = lo + (k - 1) * step + 1;
        hi = lo + k * step < hi ? lo + k * step : hi;
        lo = low;
    }
    return (unsigned)lo;
}

// V = 8: a lane's columns are neighbours; V = 1: 32 apart
template <int V> __device__ __forceinline__ int column_of(int lane, int i) { return V == 8 ? lane * 8 : lane + 32 * i; }

template <class T, int V>
struct RowPiece {
    Piece<T, V> p[8 / V];
    __device__ __forceinline__ void load(const T *__restrict__ row, int lane, int columns)
    {
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            p[i].zero();
            if (column_of<V>(lane, i) < columns) p[i].load(row + column_of<V>(lane, i));
        }
    }
    __device__ __forceinline__ void add_to(float (&a)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            float v[V];
            p[i].get(v);
#pragma unroll
            for (int j = 0; j < V; ++j) a[i * V + j] += v[j];
        }
    }
};

// the finished sum of a row
template <int V>
__device__ __forceinline__ void write_row(const Sums &P, unsigned row, int c0, int lane, int columns, const float (&a)[8], bool any)
{
    if (P.accumulate && !any) return;
    const int64_t at = (int64_t)row * P.ds + c0;
#pragma unroll
    for (int i = 0; i < 8 / V; ++i) {
        const int c = column_of<V>(lane, i);
        if (c >= columns) continue;
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = any ? a[i * V + j] * P.factor : 0.f;
        auto store = [&](auto *out) {
            using O = typename std::remove_pointer<decltype(out)>::type;
            Piece<O, V> o;
            if (P.accumulate) {
                float old[V];
                o.load(out + at + c);
                o.get(old);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] += old[j];
            }
            o.set(v);
            o.store(out + at + c);
        };
        if (P.type == TAD_F32) store(static_cast<float *>(P.dtable));
        else if (P.type == TAD_BF16) store(static_cast<__nv_bfloat16 *>(P.dtable));
        else store(static_cast<__half *>(P.dtable));
    }
}

// partial sums: eight floats a lane, `place` = segment and slice
__device__ __forceinline__ void put_part(float *to, size_t place, int lane, const float (&a)[8])
{
    Piece<float, 8> o;
    o.set(a);
    o.store(to + place * SLICE + lane * 8);
}

template <class T, int V>
__global__ void __launch_bounds__(NT)
tad_embed_sums_kernel(const Sums P)
{
    tad_wait_previous();
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * (NT / 32) + (threadIdx.x >> 5);
    const unsigned s = (unsigned)(unit / P.slices), slice = (unsigned)(unit - (int64_t)s * P.slices);
    if (s >= P.segments) return;
    const int c0 = (int)slice * SLICE, columns = min(SLICE, P.width - c0);
    const int64_t items = (int64_t)P.n + P.n_table, d0 = s * P.each, d1 = min(items, d0 + P.each);
    if (d0 >= items) {
        if (slice == 0 && lane == 0) P.cuts[s] = Cut{P.n_table, 0};
        return;
    }
    unsigned i = tokens_before(P.keys, P.n, P.n_table, d0), j = (unsigned)(d0 - i);
    const unsigned first = j;
    bool open = i > 0 && j < P.n_table && P.keys[i - 1] == j, ends = false, any = false;
    const bool opened = open;
    const T *__restrict__ dy = static_cast<const T *>(P.dy) + c0;
    float a[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = 0.f;
    int64_t left = d1 - d0;
    auto end_row = [&] {
        if (open) {
            put_part(P.head, (size_t)s * P.slices + slice, lane, a);
            ends = true;
            open = false;
        } else write_row<V>(P, j, c0, lane, columns, a, any);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = 0.f;
        any = false;
        ++j;
        --left;
    };
    while (left > 0 && j < P.n_table) {
        // the next 32 tokens; behind the last one the keys of no row
        const unsigned key = i + lane < P.n ? P.keys[i + lane] : 0xffffffffu;
        const unsigned at = i + lane < P.n ? P.at[i + lane] : 0;
        unsigned used = 0;
        while (left > 0 && j < P.n_table && used < 32) {
            // AHEAD tokens of this segment, their rows under way before the first is added
            RowPiece<T, V> p[AHEAD];
            unsigned k[AHEAD];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                k[q] = __shfl_sync(0xffffffffu, key, used + q);
                const unsigned t = __shfl_sync(0xffffffffu, at, used + q);
                const bool here = k[q] < P.n_table && (int64_t)q + (k[q] - j) < left;        // (row ends up to it and tokens before it)
                p[q].load(dy + (int64_t)t * P.dys, lane, here ? columns : 0);
            }
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                const unsigned stop = min(k[q], P.n_table);
                while (left > 0 && j < stop) end_row();
                if (left > 0 && j < P.n_table) {
                    p[q].add_to(a);
                    any = true;
                    ++used;
                    --left;
                }
            }
        }
        i += used;
    }
    // the row that is open at the end
    if (any) put_part(P.tail, (size_t)s * P.slices + slice, lane, a);
    if (slice == 0 && lane == 0) P.cuts[s] = Cut{first, (opened ? OPEN : 0u) | (ends ? ENDS : 0u)};
}

// One block a segment: the row that ends here and began in an earlier segment is the sum of the tails from there on and this segment's head.
template <int V>
__global__ void __launch_bounds__(NT)
tad_embed_join_kernel(const Sums P)
{
    __shared__ float part[NT / 32][SLICE];
    tad_wait_previous();
    const unsigned s = blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Cut cut = P.cuts[s];
    if (cut.state != (OPEN | ENDS)) return;
    // the segment that the row begins in: the last one before s that does not begin inside it
    unsigned b = s;
    for (;;) {
        const bool inside = b > lane && P.cuts[b - 1 - lane].state == OPEN && P.cuts[b - 1 - lane].first_row == cut.first_row;
        const unsigned k = __ffs(~__ballot_sync(0xffffffffu, inside)) - 1;                  // (all 32 inside: 0xffffffff)
        if (k < 32) { b -= k + 1; break; }
        b -= 32;
    }
    const unsigned count = s - b;                              // tails of the segments b .. s - 1
    for (unsigned slice = 0; slice < P.slices; ++slice) {
        const int c0 = (int)slice * SLICE, columns = min(SLICE, P.width - c0);
        float a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = 0.f;
        const unsigned lo = (unsigned)((unsigned long long)count * warp / (NT / 32)), hi = (unsigned)((unsigned long long)count * (warp + 1) / (NT / 32));
#pragma unroll 4
        for (unsigned q = b + lo; q < b + hi; ++q) {
            Piece<float, 8> p;
            float v[8];
            p.load(P.tail + ((size_t)q * P.slices + slice) * SLICE + lane * 8);
            p.get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] += v[e];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) part[warp][lane * 8 + e] = a[e];
        __syncthreads();
        if (warp != 0) continue;
        for (int w = 1; w < NT / 32; ++w)
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] += part[w][lane * 8 + e];
        Piece<float, 8> p;
        float v[8];
        p.load(P.head + ((size_t)s * P.slices + slice) * SLICE + lane * 8);
        p.get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] += v[e];
        write_row<V>(P, cut.first_row, c0, lane, columns, a, true);
    }
}

// ---- host ----

struct Layout {
    unsigned segments, slices;
    int64_t each;
    size_t keys, parts, cuts, total;       // bytes of one of the four arrays of the sort, of one plane of partial sums, of the cuts
};
Layout layout_of(int64_t n, int64_t n_table, int64_t width)
{
    auto pad = [](size_t b) { return (b + 255) & ~size_t(255); };
    Layout l{};
    l.slices = (unsigned)((width + SLICE - 1) / SLICE);
    const int64_t items = n + n_table, warps = (int64_t)SMS * 48;
    l.segments = (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + 15) / 16, (warps + l.slices - 1) / l.slices));
    l.each = (items + l.segments - 1) / l.segments;
    l.keys = pad((size_t)n * 4);
    l.parts = pad((size_t)l.segments * l.slices * SLICE * 4);
    l.cuts = pad((size_t)l.segments * sizeof(Cut));
    l.total = n > 0 ? 4 * l.keys + 2 * l.parts + l.cuts : 0;
    return l;
}

tad_status check_tokens(const char *what, const void *tokens, int32_t bits, int64_t n, int64_t n_table)
{
    if (bits != 32 && bits != 64) return bad(std::string(what) + ": tokens have 32 or 64 bits");
    if (n_table < 0) return bad(std::string(what) + ": negative size");
    if (n_table >= MAX_ROWS) { tad::set_error(std::string(what) + ": 2^31 table rows and more"); return TAD_ERR_UNSUPPORTED; }
    if (n > 0 && (!tokens || reinterpret_cast<uintptr_t>(tokens) % (bits / 8))) return bad(std::string(what) + ": tokens NULL or not aligned");
    return TAD_OK;
}

template <class S, class T>
cudaError_t embed_forward(const Tokens &tok, int64_t n, const tad_rows *table, int64_t width, float factor, const tad_rows *y, cudaStream_t stream)
{
    const bool eights = width % 8 == 0 && by_eights(table) && by_eights(y);
    const int64_t pieces = eights ? width / 8 : width;
    int log = 0;
    while (log < 8 && (int64_t(1) << log) < pieces) ++log;
    const int64_t chunks = (pieces + (1 << log) - 1) >> log, rows = ROWS * (NT >> log), blocks = (n + rows - 1) / rows * chunks;
    if (blocks >= MAX_ROWS) return cudaErrorInvalidValue;
    return tad_launch(eights ? tad_embed_forward_kernel<S, T, 8> : tad_embed_forward_kernel<S, T, 1>, (unsigned)blocks, NT, 0, stream, tok, n,
                      static_cast<const S *>(table->data), table->stride, (int)width, factor, static_cast<T *>(y->data), y->stride, log, (unsigned)chunks);
}

// rows without tokens only
__global__ void __launch_bounds__(NT)
tad_embed_zero_kernel(void *out, int type, int64_t stride, int64_t n_rows, int width)
{
    tad_wait_previous();
    for (int64_t r = blockIdx.x; r < n_rows; r += gridDim.x)
        for (int c = threadIdx.x; c < width; c += NT) put_element(out, type, r * stride + c, 0.f);
}

}  // namespace

extern "C" {

tad_status tad_embed_forward(const void *tokens, int32_t token_bits, int64_t n_tokens, const tad_rows *table, int64_t n_table,
                             int64_t width, float factor, const tad_rows *y, void *cuda_stream)
{
    tad_status st;
    if ((st = check_sizes("embed_forward", n_tokens, width)) || (st = check_tokens("embed_forward", tokens, token_bits, n_tokens, n_table)) ||
        (st = check_rows("embed_forward: table", table, n_table, width)) || (st = check_rows("embed_forward: y", y, n_tokens, width))) return st;
    if (n_tokens == 0 || width == 0) return TAD_OK;
    const Tokens tok{tokens, token_bits, (unsigned)n_table};
    cudaError_t e = cudaSuccess;
    TAD_WITH_TYPE(table->type, S, TAD_WITH_TYPE(y->type, T, e = (embed_forward<S, T>(tok, n_tokens, table, width, factor, y, (cudaStream_t)cuda_stream))));
    return launched("embedding", e);
}

size_t tad_embed_workspace_bytes(int64_t n_tokens, int64_t n_table, int64_t width)
{
    if (n_tokens <= 0 || n_table <= 0 || width <= 0 || n_tokens >= MAX_ROWS || n_table >= MAX_ROWS || width >= MAX_WIDTH) return 0;
    return layout_of(n_tokens, n_table, width).total;
}

tad_status tad_embed_backward(const void *tokens, int32_t token_bits, int64_t n_tokens, const tad_rows *dy, int64_t n_table,
                              int64_t width, float factor, const tad_rows *dtable, int32_t accumulate, void *workspace,
                              size_t workspace_bytes, void *cuda_stream)
{
    tad_status st;
    if ((st = check_sizes("embed_backward", n_tokens, width)) || (st = check_tokens("embed_backward", tokens, token_bits, n_tokens, n_table)) ||
        (st = check_rows("embed_backward: dy", dy, n_tokens, width)) || (st = check_rows("embed_backward: dtable", dtable, n_table, width))) return st;
    if ((st = check_room("embed_backward", workspace, workspace_bytes, tad_embed_workspace_bytes(n_tokens, n_table, width)))) return st;
    if (n_table == 0 || width == 0 || (n_tokens == 0 && accumulate)) return TAD_OK;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (n_tokens == 0)
        return launched("embedding gradient", tad_launch(tad_embed_zero_kernel, (unsigned)std::min<int64_t>(n_table, 16 * SMS), NT, 0, stream, dtable->data, (int)dtable->type,
                                                         dtable->stride, n_table, (int)width));
    const Layout l = layout_of(n_tokens, n_table, width);
    char *ws = static_cast<char *>(workspace);
    unsigned *k0 = reinterpret_cast<unsigned *>(ws), *p0 = reinterpret_cast<unsigned *>(ws + l.keys), *k1 = reinterpret_cast<unsigned *>(ws + 2 * l.keys),
             *p1 = reinterpret_cast<unsigned *>(ws + 3 * l.keys);
    // digits of at most nine bits; keys run to n_table, the key of tokens outside the table
    int key_bits = 1;
    while (((uint64_t)n_table >> key_bits) != 0) ++key_bits;
    const int passes = (key_bits + 8) / 9, bits = (key_bits + passes - 1) / passes;
    const int blocks = n_tokens <= 2048 ? 1 : 8;
    const int64_t warps = (int64_t)blocks * SORT_WARPS, run = ((n_tokens + warps - 1) / warps + 31) / 32 * 32;
    static std::atomic<bool> allowed[64];
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev < 0 || dev >= 64 || !allowed[dev].load(std::memory_order_relaxed))) {
        e = cudaFuncSetAttribute(tad_embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SORT_SMEM);
        if (e == cudaSuccess && dev >= 0 && dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
    }
    if (e == cudaSuccess)
        e = tad_launch_cluster(tad_embed_sort_kernel, blocks, SORT_NT, SORT_SMEM, stream, blocks, Tokens{tokens, token_bits, (unsigned)n_table},
                               (unsigned)n_tokens, (unsigned)run, passes, bits, k0, p0, k1, p1);
    if (e != cudaSuccess) return launched("sort of the tokens", e);
    Sums P{};
    P.keys = passes & 1 ? k0 : k1; P.at = passes & 1 ? p0 : p1;
    P.dy = dy->data; P.dys = dy->stride;
    P.dtable = dtable->data; P.ds = dtable->stride; P.type = dtable->type; P.accumulate = accumulate != 0;
    P.n = (unsigned)n_tokens; P.n_table = (unsigned)n_table; P.segments = l.segments; P.slices = l.slices; P.each = l.each;
    P.width = (int)width; P.factor = factor;
    P.head = reinterpret_cast<float *>(ws + 4 * l.keys); P.tail = reinterpret_cast<float *>(ws + 4 * l.keys + l.parts);
    P.cuts = reinterpret_cast<Cut *>(ws + 4 * l.keys + 2 * l.parts);
    const bool eights = width % 8 == 0 && by_eights(dy) && by_eights(dtable);
    const unsigned grid = (unsigned)(((int64_t)l.segments * l.slices + NT / 32 - 1) / (NT / 32));
    TAD_WITH_TYPE(dy->type, T, {
        auto kernel = eights ? tad_embed_sums_kernel<T, 8> : tad_embed_sums_kernel<T, 1>;
        e = tad_launch(kernel, grid, NT, 0, stream, P);
    });
    if (e == cudaSuccess) e = tad_launch(eights ? tad_embed_join_kernel<8> : tad_embed_join_kernel<1>, l.segments, NT, 0, stream, P);
    return launched("embedding gradient", e);
}

}  // extern "C"
