// Lookup of table rows by tokens and its gradient (tad_embed_forward, tad_embed_backward).
//
//     y_t = factor E_{tok_t},        dE_v = factor sum_{t : tok_t = v} dy_t
//
// The gradient is the gather form of the derivative for an index that is data: Gamma(v) = { t : tok_t = v } comes from sorting
// the positions by token instead of from an inverse index map.  A stable radix sort keeps each row's positions in ascending
// order, so the sums have a fixed order without atomics.
//
// Both directions move bytes and are bound by memory: the gradient reads dy once (rows in sorted order, whole rows at a time)
// and writes the table's gradient once, zeros included.  Measured, bf16: lookup of 65536 different rows of 2048 83 us (6.5 TB/s), of
// 16384 different rows of 1024 13.8 us (4.9 TB/s), of as many tokens of a text, which name 6000 rows, 10.4 us (4.4 TB/s of
// memory, the repeated rows from L2); gradient of 16384 tokens into 50021 x 1024 fp32 55 us (4.3 TB/s over all four kernels), added
// to what is there 32 us; of 65536 into 128000 x 2048 260 us (5.1 TB/s), added 194.  In a captured graph the zeros follow the sort instead of
// running beside it: 67 and 284 us.
// Sorting is a chain of short steps that needs few SMs, so the rows that have no token get their zeros meanwhile; a third kernel adds
// up the others, a fourth what its warps left in parts.
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
    __device__ __forceinline__ unsigned inside(long long k) const { return k >= 0 && k < (long long)n_table ? (unsigned)k : n_table; }
    __device__ __forceinline__ unsigned key(int64_t t) const { return inside(bits == 32 ? (long long)static_cast<const int *>(p)[t] : static_cast<const long long *>(p)[t]); }
    // past the first-level cache
    __device__ __forceinline__ unsigned key_from_l2(int64_t t) const
    {
        return inside(bits == 32 ? (long long)__ldcg(static_cast<const int *>(p) + t) : __ldcg(static_cast<const long long *>(p) + t));
    }
};

// ---- forward ----

constexpr int NT = 256, ROWS = 4;

// ROWS rows of eight elements a thread; 2^log threads stand beside each other in a row
template <class S, class T>
__global__ void __launch_bounds__(NT)
tad_embed_forward_kernel(const Tokens tok, int64_t n, const S *__restrict__ table, int64_t ts, int width, float factor, T *__restrict__ y,
                         int64_t ys, int log, unsigned chunks)
{
    tad_wait_previous();
    const unsigned group = blockIdx.x / chunks, chunk = blockIdx.x - group * chunks;
    const int step = NT >> log;
    const int64_t t0 = (int64_t)group * (ROWS * step) + (threadIdx.x >> log);
    const int64_t c = ((int64_t)(chunk << log) + (threadIdx.x & ((1 << log) - 1))) * 8;
    if (c >= width) return;
    unsigned key[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) key[i] = t0 + i * step < n ? tok.key(t0 + i * step) : tok.n_table;
    Piece<S, 8> p[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        p[i].zero();
        if (key[i] < tok.n_table) p[i].load(table + (int64_t)key[i] * ts + c);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (t0 + i * step >= n) continue;
        float v[8];
        p[i].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = key[i] < tok.n_table ? v[j] * factor : 0.f;      // (zeros even where the factor is not finite)
        Piece<T, 8> o;
        o.set(v);
        o.store(y + (t0 + i * step) * ys + c);
    }
}

// Rows off 16-byte boundaries: a warp a row and 512 columns, sixteen elements a lane, 32 apart, so that every access is the lane's pointer and
// a constant (one element a thread and row: 16384 rows of 1001 bf16 35 us for 16)
constexpr int ODD = 16;
template <class S, class T>
__global__ void __launch_bounds__(NT)
tad_embed_forward_odd_kernel(const Tokens tok, int64_t n, const S *__restrict__ table, int64_t ts, int width, float factor, T *__restrict__ y,
                             int64_t ys, unsigned chunks)
{
    tad_wait_previous();
    const int64_t unit = (int64_t)blockIdx.x * (NT / 32) + (threadIdx.x >> 5), t = unit / chunks;
    if (t >= n) return;
    const int c = (int)(unit - t * chunks) * (32 * ODD) + (threadIdx.x & 31), rem = width - c;
    const unsigned key = tok.key(t);
    const bool inside = key < tok.n_table;
    const S *__restrict__ from = table + (inside ? (int64_t)key * ts : 0) + c;
    T *__restrict__ to = y + t * ys + c;
    S v[ODD];
#pragma unroll
    for (int i = 0; i < ODD; ++i) if (inside && 32 * i < rem) v[i] = from[32 * i];
#pragma unroll
    for (int i = 0; i < ODD; ++i) if (32 * i < rem) to[32 * i] = from_float<T>(inside ? to_float(v[i]) * factor : 0.f);
}

// ---- the sort ----

// One cluster of blocks sorts (key, position) by digits of at most nine bits, least digit first.  A warp owns a run of consecutive
// elements and counts its digits in shared memory; the counts of a digit are prefixed over the warps of a block, the blocks of the
// cluster (read from each other's shared memory) and the digits; then the warp walks its run again and every element knows its
// place: lanes with equal digits find each other by a vote for each bit (one instruction that matches all values takes as long as
// there are values).  One launch for the whole sort, a cluster barrier where a grid of independent blocks would need a launch:
// the arrays stay in L2.  What bounds it is the chain of its phases (16384 tokens 14 us) and, later, the scattered stores of a key and its
// position (65536 32 us, 262144 90 us on eight SMs).
constexpr int SORT_NT = 1024, SORT_WARPS = SORT_NT / 32, DIGIT_BITS = 9, DIGITS = 1 << DIGIT_BITS;
constexpr size_t SORT_SMEM = SORT_WARPS * DIGITS * 4;

// (32 registers a thread: a block of the kernel below fits beside it on an SM)
__global__ void __launch_bounds__(SORT_NT, 2)
tad_embed_sort_kernel(const Tokens tok, const unsigned n, const unsigned run, const int passes, const int bits, uint2 *s0, uint2 *s1)
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
        const uint2 *in = pass & 1 ? s0 : s1;
        uint2 *out = pass & 1 ? s1 : s0;
        const int shift = pass * bits;
        // (written by other blocks of the cluster in the pass before: not from the first-level cache)
        auto at = [&](unsigned t) { return pass == 0 ? make_uint2(tok.key(t), t) : __ldcg(in + t); };
        for (int d = lane; d < digits; d += 32) mine[d] = 0;
        __syncwarp();
#pragma unroll 4
        for (unsigned t = beg + lane; t < end; t += 32) atomicAdd(&mine[(at(t).x >> shift) & (digits - 1)], 1u);
        __syncthreads();
        const int d = threadIdx.x;
        if (d < digits) {
            unsigned a = 0;
#pragma unroll 8
            for (int w = 0; w < SORT_WARPS; ++w) { const unsigned c = counts[w * DIGITS + d]; counts[w * DIGITS + d] = a; a += c; }
            total[d] = a;
        }
        cluster.sync();
        unsigned before = 0, all = 0;
        if (d < digits)
#pragma unroll 8
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
#pragma unroll 8
            for (int w = 0; w < SORT_WARPS; ++w) counts[w * DIGITS + d] += base;
        __syncthreads();
        uint2 next = beg + lane < end ? at(beg + lane) : make_uint2(0, 0);
        for (unsigned t0 = beg; t0 < end; t0 += 32) {
            const bool live = t0 + lane < end;
            const uint2 e = next;
            if (t0 + 32 + lane < end) next = at(t0 + 32 + lane);
            const unsigned digit = (e.x >> shift) & (digits - 1);
            unsigned same = __ballot_sync(0xffffffffu, live);
#pragma unroll
            for (int b = 0; b < DIGIT_BITS; ++b) {             // (bits behind the digit's are zero in all lanes)
                const bool one = digit >> b & 1;
                const unsigned ones = __ballot_sync(0xffffffffu, one);
                same &= one ? ones : ~ones;
            }
            const unsigned lower = __popc(same & ((1u << lane) - 1));
            if (live) out[mine[digit] + lower] = e;
            __syncwarp();
            if (live && lower == 0) mine[digit] += __popc(same);
            __syncwarp();
        }
        cluster.sync();
    }
}

// ---- zeros ----

// Zeros into the rows that no token names, a share of consecutive rows a block.  The block reads all tokens for that: 4 bytes a token and
// block out of L2, next to the share's rows themselves.  It runs beside the sort, which has waited for the kernels before both
// by the time that this one starts (its blocks let it start behind their own wait), and waits for the sort at its end, so
// that who waits for this kernel has waited for both.  Its own wait is what would make earlier kernels' writes visible to its first-level caches,
// so it reads the tokens from L2, where the sort's wait has them.  (105000 rows of 2048 fp32 158 us, 5.4 TB/s.)
constexpr int CLEAR_NT = 1024;
constexpr unsigned MAP_ROWS = 32768;                           // rows whose use is noted at a time, a bit each

__global__ void __launch_bounds__(CLEAR_NT)
tad_embed_clear_kernel(const Tokens tok, const unsigned n, const int64_t each, unsigned char *dtable, const int64_t stride, const int64_t row_bytes,
                       const bool beside)
{
    __shared__ unsigned map[MAP_ROWS / 32];
    if (!beside) tad_wait_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t first = blockIdx.x * each, last = min(first + each, (int64_t)tok.n_table);
    for (int64_t r0 = first; r0 < last; r0 += MAP_ROWS) {
        const unsigned rows = (unsigned)min((int64_t)MAP_ROWS, last - r0);
        __syncthreads();
        for (unsigned i = threadIdx.x; i < (rows + 31) / 32; i += CLEAR_NT) map[i] = 0;
        __syncthreads();
#pragma unroll 4
        for (int64_t t = threadIdx.x; t < n; t += CLEAR_NT) {
            const int64_t at = (int64_t)tok.key_from_l2(t) - r0;
            if (at >= 0 && at < rows) {
                const unsigned bit = 1u << (at & 31);
                if (!(*(volatile unsigned *)&map[at >> 5] & bit)) atomicOr(&map[at >> 5], bit);
            }
        }
        __syncthreads();
        for (unsigned i = warp; i < rows; i += CLEAR_NT / 32) {
            if (map[i >> 5] >> (i & 31) & 1) continue;
            unsigned char *to = dtable + (r0 + i) * stride;
            // whole sectors from the row's first boundary of 32 bytes on, two bytes a lane before and behind them
            const int64_t head = min(row_bytes, (int64_t)(-reinterpret_cast<uintptr_t>(to) & 31)), body = (row_bytes - head) & ~int64_t(31);
            if (lane * 2 < head) *reinterpret_cast<unsigned short *>(to + lane * 2) = 0;
            for (int64_t b = head + lane * 32; b < head + body; b += 1024)
                asm volatile("st.global.v8.b32 [%0], {%1,%1,%1,%1,%1,%1,%1,%1};" ::"l"(to + b), "r"(0) : "memory");
            if (lane * 2 < row_bytes - head - body) *reinterpret_cast<unsigned short *>(to + head + body + lane * 2) = 0;
        }
    }
    if (beside) tad_wait_previous();
}

// ---- the sums ----

// The sorted tokens are cut into segments of equal length, so a token that is half of the batch leaves no warps idle.  A warp owns a
// segment in 256 columns and adds up the rows of dy of one token after the other.  A token whose positions begin in one segment
// and end in another leaves a partial sum in each: `tail` of the segments that it does not end in, `head` of the one it ends in;
// tad_embed_join_kernel adds them up in order.  About 90 instructions a position and slice bound it beside the memory: 65536 tokens of
// 2048 bf16, 23000 rows written, 92 us (5 TB/s).
constexpr int SLICE = 256;
// rows of dy that a warp has under way: about as many as three blocks an SM have registers for (with pieces of eight the builds spill 24 to 60 bytes
// a thread, with single elements 4)
template <class T, int V> constexpr int AHEAD = V == 8 && sizeof(T) == 2 ? 8 : 4;
constexpr int SUM_BLOCKS = 3;

struct Cut {
    unsigned first_row;      // the token that the segment begins with
    unsigned state;          // OPEN: positions of it lie in segments before;  ENDS: its last one lies in this segment
};
constexpr unsigned OPEN = 1, ENDS = 2;

struct Sums {
    const uint2 *sorted;                                   // token, position
    const void *dy;
    int64_t dys;
    void *dtable;
    int64_t ds;
    int accumulate;
    unsigned n, n_table, segments, slices, each;           // each: positions of a segment
    int width;
    float factor;
    float *head, *tail;
    Cut *cuts;
};

// Eight columns a lane: V = 8, neighbours; V = 1, 32 apart.  A piece of a row of dy, or the sums (two columns an instruction).
template <int V> __device__ __forceinline__ constexpr int place(int i) { return V == 8 ? 0 : 32 * i; }
template <int V> __device__ __forceinline__ int first_column(int lane) { return V == 8 ? lane * 8 : lane; }

template <class T, int V>
struct RowPiece {
    Piece<T, V> p[8 / V];
    // from the lane's first column on; whole: all of the slice's columns exist
    __device__ __forceinline__ void load(const T *__restrict__ at, int rem, bool whole)
    {
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            if (whole) p[i].load(at + place<V>(i));
            else {
                p[i].zero();
                if (place<V>(i) < rem) p[i].load(at + place<V>(i));
            }
        }
    }
    __device__ __forceinline__ void add_to(float2 (&a)[4]) const
    {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            float f[V];
            p[i].get(f);
#pragma unroll
            for (int j = 0; j < V; ++j) v[i * V + j] = f[j];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = __fadd2_rn(a[j], make_float2(v[2 * j], v[2 * j + 1]));
    }
};
__device__ __forceinline__ void clear(float2 (&a)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = make_float2(0.f, 0.f);
}

// the finished sum of a row; to: the lane's first column of the slice in row 0
template <class O, int V>
__device__ __forceinline__ void write_row(const Sums &P, O *__restrict__ to, unsigned row, int rem, const float2 (&a)[4])
{
    O *at = to + (int64_t)row * P.ds;
#pragma unroll
    for (int i = 0; i < 8 / V; ++i) {
        if (place<V>(i) >= rem) continue;
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = ((i * V + j) & 1 ? a[(i * V + j) / 2].y : a[(i * V + j) / 2].x) * P.factor;
        Piece<O, V> o;
        if (P.accumulate) {
            float old[V];
            o.load(at + place<V>(i));
            o.get(old);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] += old[j];
        }
        o.set(v);
        o.store(at + place<V>(i));
    }
}

// partial sums: eight floats a lane, `part` = segment and slice
__device__ __forceinline__ float *part_at(float *parts, size_t part, int lane) { return parts + part * SLICE + lane * 8; }
__device__ __forceinline__ void put_part(float *to, const float2 (&a)[4])
{
    Piece<float, 8> o;
    o.a = make_float4(a[0].x, a[0].y, a[1].x, a[1].y);
    o.b = make_float4(a[2].x, a[2].y, a[3].x, a[3].y);
    o.store(to);
}

template <class T, class O, int V>
__global__ void __launch_bounds__(NT, SUM_BLOCKS)
tad_embed_sums_kernel(const Sums P)
{
    constexpr int A = AHEAD<T, V>;
    tad_wait_previous();
    const int lane = threadIdx.x & 31;
    const unsigned unit = blockIdx.x * (NT / 32) + (threadIdx.x >> 5), s = unit / P.slices, slice = unit - s * P.slices;
    if (s >= P.segments) return;
    const int column = (int)slice * SLICE + first_column<V>(lane), rem = P.width - column;
    const bool whole = (int)slice * SLICE + SLICE <= P.width;
    const unsigned beg = (unsigned)min((unsigned long long)P.n, (unsigned long long)s * P.each), end = (unsigned)min((unsigned long long)P.n, (unsigned long long)beg + P.each);
    unsigned row = beg < end ? P.sorted[beg].x : P.n_table;
    const unsigned first = row;
    bool open = beg > 0 && row < P.n_table && P.sorted[beg - 1].x == row, ends = false;
    const bool opened = open;
    const T *__restrict__ dy = static_cast<const T *>(P.dy) + column;
    O *__restrict__ out = static_cast<O *>(P.dtable) + column;
    float2 a[4];
    clear(a);
    // the sum of `row` is complete
    auto close = [&] {
        if (open) {
            put_part(part_at(P.head, (size_t)s * P.slices + slice, lane), a);
            ends = true;
            open = false;
        } else write_row<O, V>(P, out, row, rem, a);
        clear(a);
    };
    // (tokens outside the table are sorted to the end)
    auto positions = [&](unsigned i) { return i < end ? P.sorted[i] : make_uint2(P.n_table, 0); };
    uint2 next = positions(beg + lane);
    for (unsigned i = beg; i < end && row < P.n_table; i += 32) {
        const uint2 here = next;
        next = positions(i + 32 + lane);
        const int count = (int)min(32u, end - i);
#pragma unroll 1
        for (int u = 0; u < count; u += A) {
            // some positions, their rows under way before the first is added (behind the segment's end: row 0 once more, not added)
            RowPiece<T, V> p[A];
            unsigned k[A];
#pragma unroll
            for (int q = 0; q < A; ++q) {
                k[q] = __shfl_sync(0xffffffffu, here.x, u + q);
                p[q].load(dy + (int64_t)__shfl_sync(0xffffffffu, here.y, u + q) * P.dys, rem, whole);
            }
#pragma unroll
            for (int q = 0; q < A; ++q) {
                if (u + q >= count) continue;
                if (k[q] != row) {
                    if (row < P.n_table) close();
                    row = k[q];
                }
                if (row < P.n_table) p[q].add_to(a);
            }
        }
    }
    // the row that is open at the end
    if (row < P.n_table) {
        if (end < P.n && P.sorted[end].x == row) put_part(part_at(P.tail, (size_t)s * P.slices + slice, lane), a);
        else close();
    }
    if (slice == 0 && lane == 0) P.cuts[s] = Cut{first, (opened ? OPEN : 0u) | (ends ? ENDS : 0u)};
}

// The token that ends in segment s and began in an earlier one is the sum of the tails from there on and the head of s.  A warp a segment
// and slice; where there are many tails, the warps of the block share them (the slices of a segment lie in different blocks then).
constexpr unsigned MANY = 16;

template <class O, int V>
__global__ void __launch_bounds__(NT)
tad_embed_join_kernel(const Sums P)
{
    constexpr int WARPS = NT / 32;
    __shared__ float part[WARPS][SLICE];
    __shared__ unsigned shared_first[WARPS];                   // where the block shares the work: the segment that the row begins in
    tad_wait_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto add = [&](float2 (&a)[4], unsigned lo, unsigned hi, unsigned s, unsigned slice) {
        clear(a);
#pragma unroll 4
        for (unsigned q = lo; q < hi; ++q) {
            RowPiece<float, 8> p;
            p.load(part_at(q < s ? P.tail : P.head, (size_t)q * P.slices + slice, lane), 8, true);
            p.add_to(a);
        }
    };
    auto write = [&](const float2 (&a)[4], unsigned row, unsigned slice) {
        const int column = (int)slice * SLICE + first_column<V>(lane);
        write_row<O, V>(P, static_cast<O *>(P.dtable) + column, row, P.width - column, a);
    };
    const unsigned unit0 = blockIdx.x * WARPS, unit = unit0 + warp, slice = unit / P.segments, s = unit - slice * P.segments;
    const Cut cut = slice < P.slices ? P.cuts[s] : Cut{0, 0};
    bool many = false;
    float2 a[4];
    if (cut.state == (OPEN | ENDS)) {
        // the segment that the row begins in: the last one before s that does not begin inside it
        unsigned b = s;
        for (;;) {
            const bool inside = b > lane && P.cuts[b - 1 - lane].state == OPEN && P.cuts[b - 1 - lane].first_row == cut.first_row;
            const unsigned k = __ffs(~__ballot_sync(0xffffffffu, inside)) - 1;              // (all 32 inside: 0xffffffff)
            if (k < 32) { b -= k + 1; break; }
            b -= 32;
        }
        many = s - b > MANY;
        if (many) { if (lane == 0) shared_first[warp] = b; }
        else {
            add(a, b, s + 1, s, slice);
            write(a, cut.first_row, slice);
        }
    }
    unsigned todo = 0;
    if (!__syncthreads_or(many)) return;
    __shared__ unsigned flags[WARPS];
    if (lane == 0) flags[warp] = many;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; ++w) todo |= flags[w] << w;
    for (int w = 0; w < WARPS; ++w) {
        if (!(todo >> w & 1)) continue;
        const unsigned sl = (unit0 + w) / P.segments, su = unit0 + w - sl * P.segments, b = shared_first[w];
        const unsigned long long count = su + 1 - b;
        add(a, b + (unsigned)(count * warp / WARPS), b + (unsigned)(count * (warp + 1) / WARPS), su, sl);
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<float2 *>(&part[warp][lane * 8 + 2 * e]) = a[e];
        __syncthreads();
        if (warp == 0) {
#pragma unroll
            for (int q = 1; q < WARPS; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) a[e] = __fadd2_rn(a[e], *reinterpret_cast<const float2 *>(&part[q][lane * 8 + 2 * e]));
            write(a, P.cuts[su].first_row, sl);
        }
        __syncthreads();
    }
}

// ---- host ----

struct Layout {
    unsigned segments, slices, each;
    size_t sorted, parts, cuts, total;     // bytes of one of the two arrays of the sort, of one plane of partial sums, of the cuts
};
Layout layout_of(int64_t n, int64_t width)
{
    auto pad = [](size_t b) { return (b + 255) & ~size_t(255); };
    Layout l{};
    l.slices = (unsigned)((width + SLICE - 1) / SLICE);
    // warps for all SMs, eight positions each at least (a segment's partial sums cost as much as two)
    const int64_t warps = (int64_t)SMS * SUM_BLOCKS * (NT / 32), segments = std::max<int64_t>(1, std::min<int64_t>((n + 7) / 8, (warps + l.slices - 1) / l.slices));
    l.each = (unsigned)((n + segments - 1) / segments);
    l.segments = (unsigned)((n + l.each - 1) / l.each);
    l.sorted = pad((size_t)n * sizeof(uint2));
    l.parts = pad((size_t)l.segments * l.slices * SLICE * 4);
    l.cuts = pad((size_t)l.segments * sizeof(Cut));
    l.total = 2 * l.sorted + 2 * l.parts + l.cuts;
    return l;
}

tad_status check_tokens(const char *what, const void *tokens, int32_t bits, int64_t n, int64_t n_table)
{
    if (bits != 32 && bits != 64) return bad(what, "tokens have 32 or 64 bits");
    if (n_table < 0) return bad(what, "negative size");
    if (n_table >= MAX_ROWS) return refuse(TAD_ERR_UNSUPPORTED, what, "2^31 table rows and more");
    if (n > 0 && (!tokens || reinterpret_cast<uintptr_t>(tokens) % (bits / 8))) return bad(what, "tokens NULL or not aligned");
    return TAD_OK;
}

int64_t odd_chunks(int64_t width) { return (width + 32 * ODD - 1) / (32 * ODD); }

template <class S, class T>
cudaError_t embed_forward(const Tokens &tok, int64_t n, const tad_rows *table, int64_t width, float factor, const tad_rows *y, cudaStream_t stream)
{
    const bool eights = width % 8 == 0 && by_eights(table) && by_eights(y);
    if (!eights) {
        const int64_t chunks = odd_chunks(width), blocks = (n * chunks + NT / 32 - 1) / (NT / 32);
        return tad_launch(tad_embed_forward_odd_kernel<S, T>, (unsigned)blocks, NT, 0, stream, tok, n, static_cast<const S *>(table->data), table->stride, (int)width, factor,
                          static_cast<T *>(y->data), y->stride, (unsigned)chunks);
    }
    const int64_t pieces = width / 8;
    int log = 0;
    while (log < 8 && (int64_t(1) << log) < pieces) ++log;
    const int64_t chunks = (pieces + (1 << log) - 1) >> log, rows = ROWS * (NT >> log), blocks = (n + rows - 1) / rows * chunks;
    return tad_launch(tad_embed_forward_kernel<S, T>, (unsigned)blocks, NT, 0, stream, tok, n, static_cast<const S *>(table->data), table->stride, (int)width, factor,
                      static_cast<T *>(y->data), y->stride, log, (unsigned)chunks);
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
    // more blocks than a launch has, in either form (of matrices beyond any memory)
    if (n_tokens * odd_chunks(width) >= MAX_ROWS * (NT / 32) - NT) return refuse(TAD_ERR_UNSUPPORTED, "embed_forward", "too many blocks");
    const Tokens tok{tokens, token_bits, (unsigned)n_table};
    cudaError_t e = cudaSuccess;
    TAD_WITH_TYPE(table->type, S, TAD_WITH_TYPE(y->type, T, e = (embed_forward<S, T>(tok, n_tokens, table, width, factor, y, (cudaStream_t)cuda_stream))));
    return launched("embedding", e);
}

size_t tad_embed_workspace_bytes(int64_t n_tokens, int64_t n_table, int64_t width)
{
    if (n_tokens <= 0 || n_table <= 0 || width <= 0 || n_tokens >= MAX_ROWS || n_table >= MAX_ROWS || width >= MAX_WIDTH) return 0;
    return layout_of(n_tokens, width).total;
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
    const Layout l = n_tokens ? layout_of(n_tokens, width) : Layout{};
    char *ws = static_cast<char *>(workspace);
    uint2 *s0 = reinterpret_cast<uint2 *>(ws), *s1 = reinterpret_cast<uint2 *>(ws + l.sorted);
    const Tokens tok{tokens, token_bits, (unsigned)n_table};
    // digits of at most nine bits; keys run to n_table, the key of tokens outside the table
    int key_bits = 1;
    while (((uint64_t)n_table >> key_bits) != 0) ++key_bits;
    const int passes = (key_bits + DIGIT_BITS - 1) / DIGIT_BITS, bits = (key_bits + passes - 1) / passes;
    cudaError_t e = cudaSuccess;
    // (eight: the largest cluster that every device of the kind places; few tokens are sorted by one block, without the others' barriers)
    const int cluster = n_tokens == 0 ? 0 : n_tokens <= 2048 ? 1 : 8;
    if (n_tokens) {
        static std::atomic<bool> allowed[64];
        int dev = -1;
        e = cudaGetDevice(&dev);
        if (e == cudaSuccess && (dev < 0 || dev >= 64 || !allowed[dev].load(std::memory_order_relaxed))) {
            e = cudaFuncSetAttribute(tad_embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SORT_SMEM);
            if (e == cudaSuccess && dev >= 0 && dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
        }
        const int64_t warps = (int64_t)cluster * SORT_WARPS, run = ((n_tokens + warps - 1) / warps + 31) / 32 * 32;
        if (e == cudaSuccess)
            e = tad_launch_cluster(tad_embed_sort_kernel, cluster, SORT_NT, SORT_SMEM, stream, cluster, tok, (unsigned)n_tokens, (unsigned)run, passes, bits, s0, s1);
        if (e != cudaSuccess) return launched("sort of the tokens", e);
    }
    if (!accumulate) {
        const int64_t size = (int64_t)type_size(dtable->type), stride = dtable->stride * size, row_bytes = width * size;
        // (an SM a block beside those of the sort: a share whose SM sorts too is the last to end)
        const int64_t blocks = std::min<int64_t>(SMS - cluster, (n_table + 31) / 32), each = (n_table + blocks - 1) / blocks;
        e = tad_launch(tad_embed_clear_kernel, (unsigned)blocks, CLEAR_NT, 0, stream, tok, (unsigned)n_tokens, each, static_cast<unsigned char *>(dtable->data), stride,
                       row_bytes, n_tokens > 0);
        if (e != cudaSuccess || n_tokens == 0) return launched("clearing of rows without tokens", e);
    }
    Sums P{};
    P.sorted = passes & 1 ? s0 : s1;
    P.dy = dy->data; P.dys = dy->stride;
    P.dtable = dtable->data; P.ds = dtable->stride; P.accumulate = accumulate != 0;
    P.n = (unsigned)n_tokens; P.n_table = (unsigned)n_table; P.segments = l.segments; P.slices = l.slices; P.each = l.each;
    P.width = (int)width; P.factor = factor;
    P.head = reinterpret_cast<float *>(ws + 2 * l.sorted); P.tail = reinterpret_cast<float *>(ws + 2 * l.sorted + l.parts);
    P.cuts = reinterpret_cast<Cut *>(ws + 2 * l.sorted + 2 * l.parts);
    const bool eights = width % 8 == 0 && by_eights(dy) && by_eights(dtable);
    const unsigned grid = (unsigned)(((int64_t)l.segments * l.slices + NT / 32 - 1) / (NT / 32));
    TAD_WITH_TYPE(dtable->type, O, {
        TAD_WITH_TYPE(dy->type, T, e = tad_launch(eights ? tad_embed_sums_kernel<T, O, 8> : tad_embed_sums_kernel<T, O, 1>, grid, NT, 0, stream, P));
        if (e == cudaSuccess && l.segments > 1) e = tad_launch(eights ? tad_embed_join_kernel<O, 8> : tad_embed_join_kernel<O, 1>, grid, NT, 0, stream, P);
    });
    return launched("embedding gradient", e);
}

}  // extern "C"
