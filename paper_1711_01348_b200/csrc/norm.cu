// Layer norm over rows (tad_layernorm_forward, tad_layernorm_backward).
//
//     mean = sum x / D,  rstd = (sum (x - mean)^2 / D + eps)^(-1/2),  xh = (x - mean) rstd,  y = xh w + b
//     g = dy w,  dx = rstd (g - sum g / D - xh sum (g xh) / D),  dw = sum_rows dy xh,  db = sum_rows dy
//
// Both passes read every element once and are bound by memory.  A row is held in registers, sixteen elements a thread, by a group of
// 1 to 16 warps (of the forward pass, 32) or, in longer rows, by a cluster of such groups; a group walks over the rows that are its share.  Rows of
// whole 16-byte pieces come by bulk copies into a ring of shared memory, two to four rows ahead (32 KB of rows under way a block of the
// forward pass, 128 KB of the backward pass): prefetched into registers instead they take those that a second and third block
// an SM need (8192 x 4096 fp32, forward / backward: 51 / 83 us for 48 / 69).  Other rows are loaded an element at a time, one row ahead.  The
// variance is the mean of the squared deviations of the registers (no difference of large sums).  Weights stay in registers
// over all rows.  The backward pass keeps its share of dw and db there too and writes them once a block, as a plane of partial
// sums; a second kernel adds the planes up in a fixed order.  Rows longer than a cluster holds are read twice or three times.
// Measured, 8192 x 4096: fp32 forward 43 us, backward 67 (6.2, 6.0 TB/s); bf16 26, 40 (5.2, 5.0 TB/s: of the backward pass the rows take 32, which
// is the memory's rate, its start 2, the join of the partial sums in a block and of the blocks 1 and 2.7).
#include <cooperative_groups.h>

#include <atomic>

#include "rows.cuh"

tad_status tad_launch_pack8(const tad_rows *x, int64_t n_rows, int64_t width, const tad_packed *out, cudaStream_t stream);

std::atomic<int> tadr::lost_waits{0};

namespace {

using namespace tadr;
namespace cg = cooperative_groups;

// Threads of a block: forward 256, three blocks an SM (80 registers a thread); backward 512, one (128).  Elements of a row in a thread's
// registers (E): sixteen; eight where the backward pass loads single elements, whose next row lies in registers as well (with sixteen they
// spill, and what is spilled is waited for at once: 5003 x 1001 fp32 22 us for 17).
constexpr int FORWARD_BLOCK = 256, FORWARD_BLOCKS = 3, BACKWARD_BLOCK = 512, FORWARD_E = 16;
template <int V> constexpr int BACKWARD_E = V == 8 ? 16 : 8;
// Rows that a block of 1024 threads holds: sixteen elements a thread, of 16-bit types thirty-two (four rows of 8192 at a time, not two).
constexpr int WIDE_BLOCK = 1024;
template <class T> constexpr int WIDE_E = sizeof(T) == 2 ? 32 : 16;
constexpr int MAX_CLUSTER = 8;
constexpr int HELD = FORWARD_BLOCK * FORWARD_E * MAX_CLUSTER;      // longest row that a cluster holds
constexpr int LARGE = 1024, SMALL = 256;   // threads of a block of the kernels for longer rows

// source type of a packed matrix
struct Packed8 {};

struct Params {
    const void *x, *dy, *w, *b;
    void *y, *dx;
    const uint8_t *q, *scale;
    uint8_t *kq, *kscale;
    int64_t xs, dys, ys, dxs, qs, ss, kqs, kss;
    float *mean, *rstd, *planes;
    int64_t n_rows;
    int width, w_type, b_type, y_type, dx_type;
    int group;                             // threads of a group
    float eps, inv_width;
    int lost;                              // waits count as run out (tests)
};

// How rows are divided: a warp a row, a group of warps, a cluster of groups (a block each).
enum { BY_WARP, BY_GROUP, BY_CLUSTER };

// A thread's E elements lie in the 32 E columns of its warp: V = 8, pieces of eight, 256 columns apart; V = 1, 32 apart.  So every access of
// a row is the thread's pointer and a constant, and the warp's accesses are contiguous.  Piece i exists where place(i) < rem, the columns
// from the thread's first one to the end of the row.
template <int V> struct Of {
    __device__ __forceinline__ static constexpr int place(int i) { return V == 8 ? i * 256 : i * 32; }
    // column of element e behind the thread's first
    __device__ __forceinline__ static constexpr int column(int e) { return place(e / V) + e % V; }
};

template <class T, int V, int E>
struct Held {
    Piece<T, V> p[E / V];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < E / V; ++i) p[i].zero();
    }
    // (pieces that do not exist keep their zeros)
    __device__ __forceinline__ void fetch(const T *__restrict__ at, int rem)
    {
#pragma unroll
        for (int i = 0; i < E / V; ++i) if (Of<V>::place(i) < rem) p[i].load(at + Of<V>::place(i));
    }
    __device__ __forceinline__ void get(float (&v)[E]) const
    {
#pragma unroll
        for (int i = 0; i < E / V; ++i) {
            float f[V];
            p[i].get(f);
#pragma unroll
            for (int j = 0; j < V; ++j) v[i * V + j] = f[j];
        }
    }
};

// E elements of a vector whose type is known at run time; behind the row zeros
template <class T, int V, int E>
__device__ __forceinline__ void load_held(float (&v)[E], const T *p, int rem)
{
    Held<T, V, E> h;
    h.zero();
    h.fetch(p, rem);
    h.get(v);
}
template <int V, int E>
__device__ __forceinline__ void load_vector(float (&v)[E], const void *p, int type, int c, int rem, float none)
{
    if (!p) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = none;
    } else if (V != 1 && reinterpret_cast<uintptr_t>(p) % 16 != 0) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = Of<V>::place(e / V) < rem ? element(p, type, c + Of<V>::column(e)) : 0.f;
    } else if (type == TAD_F32) load_held<float, V, E>(v, static_cast<const float *>(p) + c, rem);
    else if (type == TAD_BF16) load_held<__nv_bfloat16, V, E>(v, static_cast<const __nv_bfloat16 *>(p) + c, rem);
    else load_held<__half, V, E>(v, static_cast<const __half *>(p) + c, rem);
}

template <class O, int V, int E>
__device__ __forceinline__ void store_held(O *at, int rem, const float (&v)[E])
{
#pragma unroll
    for (int i = 0; i < E / V; ++i) {
        if (Of<V>::place(i) >= rem) continue;
        float f[V];
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = v[i * V + j];
        Piece<O, V> o;
        o.set(f);
        o.store(at + Of<V>::place(i));
    }
}
template <int V, int E>
__device__ __forceinline__ void store_typed(void *base, int type, int64_t at, int rem, const float (&v)[E])
{
    if (type == TAD_F32) store_held<float, V, E>(static_cast<float *>(base) + at, rem, v);
    else if (type == TAD_BF16) store_held<__nv_bfloat16, V, E>(static_cast<__nv_bfloat16 *>(base) + at, rem, v);
    else store_held<__half, V, E>(static_cast<__half *>(base) + at, rem, v);
}

// two elements by one instruction (elements 2 j and 2 j + 1 of a thread)
template <int E> struct Pairs {
    float2 p[E / 2];
    __device__ __forceinline__ void set(const float (&v)[E])
    {
#pragma unroll
        for (int j = 0; j < E / 2; ++j) p[j] = make_float2(v[2 * j], v[2 * j + 1]);
    }
    __device__ __forceinline__ void get(float (&v)[E]) const
    {
#pragma unroll
        for (int j = 0; j < E / 2; ++j) { v[2 * j] = p[j].x; v[2 * j + 1] = p[j].y; }
    }
};
// a value of the pieces that exist, zero behind the row, for elements 2 j and 2 j + 1
template <int V> __device__ __forceinline__ float2 inside(float v, int j, int rem)
{
    return make_float2(Of<V>::place(2 * j / V) < rem ? v : 0.f, Of<V>::place((2 * j + 1) / V) < rem ? v : 0.f);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// A thread whose wait has run out is lost: it waits no more, and what the data were for is NaN from here on.  What is on its way into the block's
// memory must not land there when the block, or the next one, uses that for something else: behind the loop over the rows a lost thread lingers
// (about a millisecond; copies were issued before the wait that has run out began, values of other blocks take a microsecond).  Waiting
// for each of them instead takes registers and time in the loop, 2 - 15 % of it.
constexpr long long WAIT_LIMIT = 1ll << 31;        // clocks (about a second) after which a wait gives up
__device__ __forceinline__ bool wait_once(unsigned bar, unsigned parity)
{
    unsigned ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool wait_for(unsigned bar, unsigned parity)
{
    if (wait_once(bar, parity)) return true;
    const long long begin = clock64();
    while (clock64() - begin < WAIT_LIMIT) if (wait_once(bar, parity)) return true;
    return false;
}

__device__ __forceinline__ void linger()
{
    const long long begin = clock64();
    while (clock64() - begin < (1ll << 21)) { }
}
// (hides from the compiler that a flag is not set where a wait has ended well: it would make two loops over the rows of it, 4 - 6 % slower in clusters)
__device__ __forceinline__ void keep_one_loop(bool &flag)
{
    int f = flag;
    asm volatile("" : "+r"(f));
    flag = f;
}

// Sums of N values over the threads of a group, the same bits in each of them.  A warp's sum goes into a box of shared
// memory, everybody adds the boxes up in order; two sets of boxes are used in turn, so one barrier a sum is enough.  ALONE: the group
// is the block.
template <int N, int BY, bool ALONE, int WARPS>
struct Sum {
    float (*box)[WARPS][N];                // [2], of this block
    int first, warps, id, threads;         // this group: its first warp, its warps, its barrier and its threads
    int turn;
    __device__ __forceinline__ void of(float (&v)[N])
    {
        if (BY == BY_WARP) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = warp_sum(v[k]);
            return;
        }
        // two values in five steps: the halves of the warp trade one for the other and go on with one each
        const int lane = threadIdx.x & 31, mine = N == 2 ? lane >> 4 : 0;
        float a = N == 2 && mine ? v[N - 1] : v[0];
        a += __shfl_xor_sync(0xffffffffu, N == 2 && !mine ? v[N - 1] : v[0], 16);
#pragma unroll
        for (int d = 8; d; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
        if (lane % (32 / N) == 0) box[turn][threadIdx.x >> 5][mine] = a;
        // (barriers with a number known at run time only count as all sixteen of a block: four blocks an SM)
        if (ALONE) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
        float2 both = make_float2(0.f, 0.f);                       // N = 2: the two sums; N = 1: of the even and of the odd warps
#pragma unroll
        for (int w = 0; w < WARPS; w += 2) {                       // (groups have an even number of warps)
            if (w >= warps) break;
            if (N == 2) {
                const float4 p = *reinterpret_cast<const float4 *>(&box[turn][first + w][0]);
                both = __fadd2_rn(both, __fadd2_rn(make_float2(p.x, p.y), make_float2(p.z, p.w)));
            } else both = __fadd2_rn(both, *reinterpret_cast<const float2 *>(&box[turn][first + w][0]));
        }
        if (N == 2) { v[0] = both.x; v[N - 1] = both.y; }
        else v[0] = both.x + both.y;
        turn ^= 1;
    }
};

// What the blocks of a cluster tell each other: two values a block and row go into everybody's shared memory by stores that count
// at the receiver's mbarrier.  (A cluster barrier instead would wait, as a release, for the rows just written: 8192 columns forward
// 55 us for 36 - 42.)
struct Exchange {
    float2 far[2][MAX_CLUSTER];
    unsigned long long bar[2];
};
struct Trade {
    Exchange *ex;
    unsigned blocks, rank, count;
    bool lost;                             // a lost thread sends nothing, a lost first thread arms no barrier: then nobody takes one row's values for another's
    __device__ __forceinline__ void start(const Params &P, Exchange *e)
    {
        ex = e; count = 0; lost = P.lost;
        cg::cluster_group cluster = cg::this_cluster();
        blocks = cluster.num_blocks();
        rank = cluster.block_rank();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"((unsigned)__cvta_generic_to_shared(&ex->bar[i])) : "memory");
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        cluster.sync();
    }
    // the values of all blocks, in order.  A barrier of the block lies between two trades: a block writes its values n + 2 behind everybody's
    // values n + 1, which are sent behind that barrier and so behind the reads of the values n.  lost: they are not the values.
    __device__ __forceinline__ const float2 *with_all(float a, float b)
    {
        const unsigned turn = count & 1, parity = (count >> 1) & 1, bar = (unsigned)__cvta_generic_to_shared(&ex->bar[turn]);
        ++count;
        if (threadIdx.x == 0 && !lost) asm volatile("{ .reg .b64 t; mbarrier.arrive.expect_tx.shared::cta.b64 t, [%0], %1; }" ::"r"(bar), "r"(blocks * 8) : "memory");
        if (threadIdx.x < blocks && !lost) {
            unsigned to, at;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((unsigned)__cvta_generic_to_shared(&ex->far[turn][rank])), "r"(threadIdx.x));
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(bar), "r"(threadIdx.x));
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(to), "r"(__float_as_uint(a)), "r"(__float_as_uint(b)), "r"(at) : "memory");
        }
        if (!lost) lost = !wait_for(bar, parity);
        keep_one_loop(lost);
        return ex->far[turn];
    }
    // no block leaves while another one may still write into it; a lost one has not seen all values arrive (behind the barrier all are sent)
    __device__ __forceinline__ void finish()
    {
        cg::this_cluster().sync();
        if (lost) linger();
    }
};

// this thread's place: its group in the grid, the groups of the grid, its first column
template <int BY, int V, int E>
struct Place {
    int64_t row, step;
    int group, in;                         // the group in the block, the thread in the group
    int col0, col, rem;                    // first column of the block and of the thread; columns from there to the end of the row
    __device__ __forceinline__ Place(const Params &P)
    {
        const int groups = BY == BY_CLUSTER ? 1 : blockDim.x / P.group;
        group = BY == BY_CLUSTER ? 0 : threadIdx.x / P.group;
        in = threadIdx.x - group * P.group;
        if (BY == BY_CLUSTER) {
            cg::cluster_group cluster = cg::this_cluster();
            const unsigned n = cluster.num_blocks();
            row = blockIdx.x / n;
            step = gridDim.x / n;
            col0 = (int)(cluster.block_rank() * blockDim.x) * E;
        } else {
            row = (int64_t)blockIdx.x * groups + group;
            step = (int64_t)gridDim.x * groups;
            col0 = 0;
        }
        col = col0 + (in >> 5) * (32 * E) + (in & 31) * V;
        rem = P.width - col;
    }
};

template <int N, int BY, bool ALONE, int WARPS>
__device__ __forceinline__ Sum<N, BY, ALONE, WARPS> sum_of(const Params &P, float (*box)[WARPS][N])
{
    const int g = BY == BY_CLUSTER ? 0 : threadIdx.x / P.group;
    return Sum<N, BY, ALONE, WARPS>{box, g * (P.group >> 5), P.group >> 5, 1 + g, P.group, 0};
}

// ---- rows ahead ----

__device__ __forceinline__ unsigned smem_u32(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }

// The ring of a group: STAGES rows (of a block's columns) of up to two tensors, a barrier a stage that counts their bytes.  The group's first
// thread issues the copies.
template <int STAGES>
struct Ring {
    unsigned buf, bars, stage_bytes;       // this group's rows (offset in `rows`) and barriers
    unsigned char *rows;
    bool leader, lost;                     // a lost leader issues no further copies
    int at;                                // the stage of the next row
    unsigned parity;
    __device__ __forceinline__ void start(unsigned char *smem, unsigned offset, unsigned bar, unsigned bytes, bool first, bool lost_before)
    {
        rows = smem; buf = offset; bars = bar; stage_bytes = bytes; leader = first; lost = lost_before; at = 0; parity = 0;
        if (leader) {
#pragma unroll
            for (int i = 0; i < STAGES; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + 8 * i) : "memory");
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.global;" ::: "memory");          // (the rows are another kernel's plain stores)
        }
    }
    // by the leader: a row's bytes of a tensor into stage `i` at `offset`; expect() first, with the bytes of all of them
    __device__ __forceinline__ void expect(int i, unsigned bytes)
    {
        asm volatile("{ .reg .b64 t; mbarrier.arrive.expect_tx.shared::cta.b64 t, [%0], %1; }" ::"r"(bars + 8 * i), "r"(bytes) : "memory");
    }
    __device__ __forceinline__ void copy(int i, unsigned offset, const void *from, unsigned bytes)
    {
        if (bytes) asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(rows) + buf + i * stage_bytes + offset), "l"(from), "r"(bytes), "r"(bars + 8 * i) : "memory");
    }
    // by the threads of the group: zeros into the bytes of every stage that no copy writes; a barrier follows
    __device__ __forceinline__ void zeros(unsigned from, unsigned to, int in, int threads) const
    {
        for (unsigned b = from + in * 16; b < to; b += threads * 16)
#pragma unroll
            for (int i = 0; i < STAGES; ++i) *reinterpret_cast<uint4 *>(rows + buf + i * stage_bytes + b) = make_uint4(0, 0, 0, 0);
    }
    // waits for the row at the ring's head
    __device__ __forceinline__ void wait()
    {
        if (!lost) lost = !wait_for(bars + 8 * at, parity);
    }
    __device__ __forceinline__ const unsigned char *row() const { return rows + buf + at * stage_bytes; }
    __device__ __forceinline__ void advance() { if (++at == STAGES) { at = 0; parity ^= 1; } }
};

// The thread's elements of a row in the ring.  Every thread reads its places, whether they exist or not: those behind the row hold zeros
// from the start (Ring::zeros), which costs no selects where the row is read.
template <class T, int E>
__device__ __forceinline__ void read_row(Piece<T, 8> (&p)[E / 8], const T *at)
{
#pragma unroll
    for (int i = 0; i < E / 8; ++i) p[i].load(at + Of<8>::place(i));
}
template <class T, int E>
__device__ __forceinline__ void elements(float (&v)[E], const Piece<T, 8> (&p)[E / 8])
{
#pragma unroll
    for (int i = 0; i < E / 8; ++i) {
        float f[8];
        p[i].get(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i * 8 + j] = f[j];
    }
}
// ---- forward ----

template <class T> constexpr int FORWARD_STAGES = sizeof(T) == 2 ? 4 : 2;

// fp32 into 8 bits beside the pass: sixteen neighbouring threads hold a block of 128.  lost: NaNs
__device__ __forceinline__ void keep_row(const Params &P, int64_t r, int col, int rem, const float (&v)[FORWARD_E], bool lost)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float f[8], a = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) { f[j] = v[8 * i + j]; a = fmaxf(a, fabsf(f[j])); }
#pragma unroll
        for (int d = 8; d; d >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
        if (__any_sync(0xffffffffu, isinf(a))) {           // (a maximum leaves out NaNs, but not infinities)
            a = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) { a = fmaxf(a, finite_abs(f[j])); f[j] = no_infinity(f[j]); }
#pragma unroll
            for (int d = 8; d; d >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
        }
        const unsigned byte = scale_byte(a);
        const float inv = inverse_scale(byte);
        if (Of<8>::place(i) >= rem) continue;
        const int c = col + Of<8>::place(i);
        uint2 u = make_uint2(to_e4m3x2(f[0] * inv, f[1] * inv) | (to_e4m3x2(f[2] * inv, f[3] * inv) << 16), to_e4m3x2(f[4] * inv, f[5] * inv) | (to_e4m3x2(f[6] * inv, f[7] * inv) << 16));
        if (lost) u = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
        *reinterpret_cast<uint2 *>(P.kq + r * P.kqs + c) = u;
        if ((threadIdx.x & 15) == 0) P.kscale[r * P.kss + c / TAD_BLOCK8] = (uint8_t)byte;
    }
}

// V = 8: width and all row starts are whole pieces of eight.  KEEP: with the checkpoint of fp32 rows.  WIDE: rows beyond what a block of 256 holds, by
// groups of a block of up to 1024 threads with so many stages; the weights lie in shared memory, where they take no registers.  (By clusters, with an
// exchange a row, bf16: 8192 x 5120 80 us for 32.5, 8192 x 6144 80 for 34, 4096 x 8192 43 for 26, 2048 x 16384 50 for 35.  Two rows of a group at a
// time, whose sums share barriers, with sixteen elements of each a thread: 43, 56, 38.)
template <class T, int V, int BY, bool KEEP = false, int WIDE = 0>
__global__ void __launch_bounds__(WIDE ? WIDE_BLOCK : FORWARD_BLOCK, WIDE ? 1 : V == 1 ? 2 : FORWARD_BLOCKS)
tad_norm_forward_kernel(const Params P)
{
    constexpr int E = WIDE ? WIDE_E<T> : FORWARD_E, STAGES = WIDE ? WIDE : FORWARD_STAGES<T>, WARPS = (WIDE ? WIDE_BLOCK : FORWARD_BLOCK) / 32;
    __shared__ __align__(16) float box[2][WARPS][1];
    __shared__ Exchange ex;
    __shared__ unsigned long long bars[WARPS][STAGES];
    extern __shared__ __align__(128) unsigned char rows[];
    tad_wait_previous();
    Sum<1, BY, !WIDE, WARPS> sum = sum_of<1, BY, !WIDE, WARPS>(P, box);
    const Place<BY, V, E> at(P);
    int64_t r = at.row;
    const T *__restrict__ x = static_cast<const T *>(P.x);
    Held<T, 1, V == 1 ? E : 1> next;       // (V = 1)
    Ring<STAGES> ring;
    const unsigned columns = (unsigned)max(0, min(P.width - at.col0, P.group * E)), bytes = columns * (unsigned)sizeof(T);
    // the first rows are under way before anything else is done
    if constexpr (V != 1) {
        const unsigned stage = P.group * E * (unsigned)sizeof(T);
        ring.start(rows, at.group * STAGES * stage, smem_u32(&bars[at.group][0]), stage, at.in == 0, !WIDE && P.lost);      // (WIDE: a register too many)
        if (ring.leader)
            for (int i = 0; i < STAGES; ++i)
                if (r + i * at.step < P.n_rows) {
                    ring.expect(i, bytes);
                    ring.copy(i, 0, x + (r + i * at.step) * P.xs + at.col0, bytes);
                }
        ring.zeros(bytes, stage, at.in, P.group);
    } else {
        next.zero();
        if (r < P.n_rows) next.fetch(x + r * P.xs + at.col, at.rem);
    }
    Pairs<WIDE ? 2 : E> w, b;
    // WIDE: four planes of float4, weights and biases 0 .. 3 and 4 .. 7 of every eight columns
    const unsigned eights = P.group * E / 8;
    float4 *const vectors = reinterpret_cast<float4 *>(rows + (size_t)blockDim.x * E * STAGES * sizeof(T));
    if constexpr (WIDE) {
        for (unsigned c = threadIdx.x; c < eights; c += blockDim.x) {
            float f[8], g[8];
            load_vector<8, 8>(f, P.w, P.w_type, c * 8, P.width - (int)c * 8, 1.f);
            load_vector<8, 8>(g, P.b, P.b_type, c * 8, P.width - (int)c * 8, 0.f);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                vectors[h * eights + c] = make_float4(f[4 * h], f[4 * h + 1], f[4 * h + 2], f[4 * h + 3]);
                vectors[(2 + h) * eights + c] = make_float4(g[4 * h], g[4 * h + 1], g[4 * h + 2], g[4 * h + 3]);
            }
        }
    } else {
        float f[E];
        load_vector<V, E>(f, P.w, P.w_type, at.col, at.rem, 1.f);
        w.set(f);
        load_vector<V, E>(f, P.b, P.b_type, at.col, at.rem, 0.f);
        b.set(f);
    }
    Trade trade;
    if constexpr (BY == BY_CLUSTER) trade.start(P, &ex);
    else if constexpr (V != 1) __syncthreads();
    for (; r < P.n_rows; r += at.step) {
        float v[E];
        if constexpr (V != 1) {
            ring.wait();
            Piece<T, 8> p[E / 8];
            read_row<T, E>(p, reinterpret_cast<const T *>(ring.row()) + (at.col - at.col0));
            elements<T, E>(v, p);
            if constexpr (KEEP) {
                keep_one_loop(ring.lost);
                keep_row(P, r, at.col, at.rem, v, ring.lost);
            }
        } else {
            next.get(v);
            if (r + at.step < P.n_rows) next.fetch(x + (r + at.step) * P.xs + at.col, at.rem);
        }
        Pairs<E> u;
        u.set(v);
        float2 two = u.p[0];
#pragma unroll
        for (int j = 1; j < E / 2; ++j) two = __fadd2_rn(two, u.p[j]);
        float s[1] = {two.x + two.y};
        sum.of(s);
        if constexpr (V != 1) {
            // (behind the sum every thread of the group has read the row)
            if (ring.leader && !ring.lost && r + STAGES * at.step < P.n_rows) {
                ring.expect(ring.at, bytes);
                ring.copy(ring.at, 0, x + (r + STAGES * at.step) * P.xs + at.col0, bytes);
            }
            ring.advance();
        }
        // the mean, in a cluster that of the block's columns, and the squared deviations from it
        const float total = V != 1 && ring.lost ? __uint_as_float(0x7fffffffu) : s[0];          // (a row that never came)
        float mean = BY == BY_CLUSTER ? (columns ? total / (float)columns : 0.f) : total * P.inv_width;
        two = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < E / 2; ++j) {
            u.p[j] = __fadd2_rn(u.p[j], inside<V>(-mean, j, at.rem));        // (zeros behind the row deviate by nothing)
            two = __ffma2_rn(u.p[j], u.p[j], two);
        }
        s[0] = two.x + two.y;
        sum.of(s);
        if constexpr (BY == BY_CLUSTER) {
            // one exchange a row: the squares about the row's mean are those about a block's and the block's count times the squared distance
            // of the two
            const float2 *all = trade.with_all(total, s[0]);
            float sums = trade.lost ? __uint_as_float(0x7fffffffu) : 0.f, squares = 0.f;            // (a block that never came)
            for (unsigned b = 0; b < trade.blocks; ++b) sums += all[b].x;
            const float whole = sums * P.inv_width;
            for (unsigned b = 0; b < trade.blocks; ++b) {
                const int n = max(0, min(P.width - (int)(b * blockDim.x) * E, (int)blockDim.x * E));
                const float d = n ? all[b].x / (float)n - whole : 0.f;
                squares += all[b].y + (float)n * (d * d);
            }
            s[0] = squares;
            const float2 shift = make_float2(mean - whole, mean - whole);
#pragma unroll
            for (int j = 0; j < E / 2; ++j) u.p[j] = __fadd2_rn(u.p[j], shift);
            mean = whole;
        }
        const float rstd = rsqrtf(s[0] * P.inv_width + P.eps);
        if (at.col == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
        const float2 rr = make_float2(rstd, rstd);
#pragma unroll
        for (int j = 0; j < E / 2; ++j) {
            if constexpr (WIDE) {
                const unsigned place = (j >> 1 & 1) * eights + at.col / 8 + Of<8>::place(j / 4) / 8;
                const float4 ww = vectors[place], bb = vectors[2 * eights + place];
                u.p[j] = __ffma2_rn(__fmul2_rn(u.p[j], rr), j & 1 ? make_float2(ww.z, ww.w) : make_float2(ww.x, ww.y), j & 1 ? make_float2(bb.z, bb.w) : make_float2(bb.x, bb.y));
            } else u.p[j] = __ffma2_rn(__fmul2_rn(u.p[j], rr), w.p[j], b.p[j]);
        }
        u.get(v);
        store_typed<V, E>(P.y, P.y_type, r * P.ys + at.col, at.rem, v);
    }
    if constexpr (V != 1)
        if (ring.lost) linger();
    if constexpr (BY == BY_CLUSTER) trade.finish();
}

// of one value over a block of 1024 threads
template <int N>
__device__ __forceinline__ float block_sum(float v, float (*box)[N][32], int &turn, int k)
{
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) box[turn][k][threadIdx.x >> 5] = v;
    __syncthreads();
    v = warp_sum(box[turn][k][threadIdx.x & 31]);
    turn ^= 1;
    return v;
}

// rows of any length: three passes over the row, the second and third from L2
template <class T>
__global__ void __launch_bounds__(LARGE)
tad_norm_forward_long_kernel(const Params P)
{
    __shared__ float box[2][1][32];
    tad_wait_previous();
    int turn = 0;
    for (int64_t r = blockIdx.x; r < P.n_rows; r += gridDim.x) {
        const T *__restrict__ x = static_cast<const T *>(P.x) + r * P.xs;
        float a = 0.f;
#pragma unroll 8
        for (int c = threadIdx.x; c < P.width; c += LARGE) a += to_float(x[c]);
        const float mean = block_sum(a, box, turn, 0) * P.inv_width;
        a = 0.f;
#pragma unroll 8
        for (int c = threadIdx.x; c < P.width; c += LARGE) { const float d = to_float(x[c]) - mean; a += d * d; }
        const float rstd = rsqrtf(block_sum(a, box, turn, 0) * P.inv_width + P.eps);
        if (threadIdx.x == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
#pragma unroll 4
        for (int c = threadIdx.x; c < P.width; c += LARGE) {
            const float w = P.w ? element(P.w, P.w_type, c) : 1.f, b = P.b ? element(P.b, P.b_type, c) : 0.f;
            put_element(P.y, P.y_type, r * P.ys + c, fmaf((to_float(x[c]) - mean) * rstd, w, b));
        }
    }
}

// ---- backward ----

// where the input of the forward pass comes from: a matrix, or its packed form
template <class S, int V>
struct Source {
    Piece<S, V> p;
    __device__ __forceinline__ void zero() { p.zero(); }
    __device__ __forceinline__ void load(const Params &P, int64_t r, int c) { p.load(static_cast<const S *>(P.x) + r * P.xs + c); }
    __device__ __forceinline__ void get(float (&v)[V]) const { p.get(v); }
};
template <>
struct Source<Packed8, 1> {
    uint8_t q, s;
    __device__ __forceinline__ void zero() { q = 0; s = 127; }
    __device__ __forceinline__ void load(const Params &P, int64_t r, int c) { q = P.q[r * P.qs + c]; s = P.scale[r * P.ss + c / TAD_BLOCK8]; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = from_e4m3x2(q).x * scale_of(s); }
};

// V = 1: the thread's elements of the next row of the input
template <class S, int E>
struct HeldSource {
    Held<S, 1, E> h;
    __device__ __forceinline__ void zero() { h.zero(); }
    __device__ __forceinline__ void fetch(const Params &P, int64_t r, int col, int rem) { h.fetch(static_cast<const S *>(P.x) + r * P.xs + col, rem); }
    __device__ __forceinline__ void get(float (&v)[E]) const { h.get(v); }
};
template <int E>
struct HeldSource<Packed8, E> {
    uint8_t q[E], s[(E + 3) / 4];          // (four elements of a thread, 32 apart, lie in one block of 128: its first column is a multiple of 256)
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < E; ++i) q[i] = 0;
#pragma unroll
        for (int k = 0; k < (E + 3) / 4; ++k) s[k] = 127;
    }
    __device__ __forceinline__ void fetch(const Params &P, int64_t r, int col, int rem)
    {
        const uint8_t *from = P.q + r * P.qs + col, *scale = P.scale + r * P.ss + col / TAD_BLOCK8;
#pragma unroll
        for (int i = 0; i < E; ++i) if (Of<1>::place(i) < rem) q[i] = from[Of<1>::place(i)];
#pragma unroll
        for (int k = 0; k < (E + 3) / 4; ++k) if (Of<1>::place(4 * k) < rem) s[k] = scale[k];
    }
    __device__ __forceinline__ void get(float (&v)[E]) const
    {
        static_assert(E == 1 || E % 4 == 0, "whole blocks");
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = from_e4m3x2(q[i]).x * scale_of(s[i / 4]);
    }
};

// V = 8: bytes of an element in memory
template <class S> constexpr int SOURCE_BYTES = sizeof(S);
template <> constexpr int SOURCE_BYTES<Packed8> = 1;
template <class S, class T> constexpr int BACKWARD_STAGES = SOURCE_BYTES<S> + (int)sizeof(T) <= 4 ? 4 : 2;

// The block's plane (group, t, col: a thread's place): its groups are added up in order through shared memory, all elements at once (V = 8 in the ring, which nobody reads
// any more), every thread's next to its neighbour's.  (Eight elements at a time, a thread's in a row: 3.3 us for 1.)
template <int V, int E>
__device__ __forceinline__ void join_groups(const Params &P, const float (&dw)[E], const float (&db)[E], float *room, int group, int t, int col)
{
    float *plane = P.planes + (size_t)blockIdx.x * 2 * P.width;
    const int groups = blockDim.x / P.group;
    __syncthreads();
    if constexpr (V == 8) {
        float4 *to = reinterpret_cast<float4 *>(room);
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            to[q * blockDim.x + threadIdx.x] = make_float4(dw[4 * q], dw[4 * q + 1], dw[4 * q + 2], dw[4 * q + 3]);
            to[(E / 4 + q) * blockDim.x + threadIdx.x] = make_float4(db[4 * q], db[4 * q + 1], db[4 * q + 2], db[4 * q + 3]);
        }
        __syncthreads();
        for (int p = group; p < E / 4; p += groups) {
            const int c = col + Of<8>::place(p % (E / 8));
            if (c >= P.width) continue;
            float a[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int g = 0; g < groups; ++g) {
                const float4 x = to[2 * p * blockDim.x + g * P.group + t], y = to[(2 * p + 1) * blockDim.x + g * P.group + t];
                a[0] += x.x; a[1] += x.y; a[2] += x.z; a[3] += x.w; a[4] += y.x; a[5] += y.y; a[6] += y.z; a[7] += y.w;
            }
            Piece<float, 8> o;
            o.set(a);
            o.store(plane + (p < E / 8 ? 0 : (size_t)P.width) + c);
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            room[e * blockDim.x + threadIdx.x] = dw[e];
            room[(E + e) * blockDim.x + threadIdx.x] = db[e];
        }
        __syncthreads();
        for (int p = group; p < 2 * E; p += groups) {
            const int c = col + Of<1>::place(p % E);
            float a = 0.f;
            for (int g = 0; g < groups; ++g) a += room[p * blockDim.x + g * P.group + t];
            if (c < P.width) plane[(p < E ? 0 : (size_t)P.width) + c] = a;
        }
    }
}

template <class S, class T, int V, int BY>
__global__ void __launch_bounds__(BACKWARD_BLOCK, 1)
tad_norm_backward_kernel(const Params P)
{
    constexpr int E = BACKWARD_E<V>, STAGES = BACKWARD_STAGES<S, T>;
    __shared__ __align__(16) float box[2][BACKWARD_BLOCK / 32][2];
    __shared__ Exchange ex;
    __shared__ unsigned long long bars[BACKWARD_BLOCK / 32][STAGES];
    extern __shared__ __align__(128) unsigned char rows[];
    __shared__ __align__(16) float join[V == 8 || BY == BY_CLUSTER ? 1 : 2 * E * BACKWARD_BLOCK];
    tad_wait_previous();
    Sum<2, BY, BY == BY_CLUSTER, BACKWARD_BLOCK / 32> sum = sum_of<2, BY, BY == BY_CLUSTER, BACKWARD_BLOCK / 32>(P, box);
    const Place<BY, V, E> at(P);
    int64_t r = at.row;
    const T *__restrict__ dy = static_cast<const T *>(P.dy);
    constexpr bool PACKED = std::is_same<S, Packed8>::value;
    constexpr int ONE = V == 1 ? E : 1;
    HeldSource<S, ONE> nx;                 // (V = 1)
    Held<T, 1, ONE> ndy;
    Ring<STAGES> ring;                     // (V = 8)
    const unsigned columns = (unsigned)max(0, min(P.width - at.col0, P.group * E)), held = P.group * E;
    const unsigned x_bytes = PACKED ? (columns + 15) & ~15u : columns * SOURCE_BYTES<S>, dy_bytes = columns * (unsigned)sizeof(T);
    float nmean = 0.f, nrstd = 0.f;
    unsigned nscale[E / 8];                // (packed, V = 8)
    auto issue = [&](int i, int64_t row) {
        ring.expect(i, x_bytes + dy_bytes);
        if constexpr (PACKED) ring.copy(i, 0, P.q + row * P.qs + at.col0, x_bytes);
        else ring.copy(i, 0, static_cast<const S *>(P.x) + row * P.xs + at.col0, x_bytes);
        ring.copy(i, held * SOURCE_BYTES<S>, dy + row * P.dys + at.col0, dy_bytes);
    };
    // what is a few bytes a thread, one row ahead
    auto fetch = [&](int64_t row) {
        if (row >= P.n_rows) return;
        nmean = P.mean[row];
        nrstd = P.rstd[row];
        if constexpr (V == 1) {
            nx.fetch(P, row, at.col, at.rem);
            ndy.fetch(dy + row * P.dys + at.col, at.rem);
        } else if constexpr (PACKED) {
#pragma unroll
            for (int i = 0; i < E / 8; ++i) if (Of<8>::place(i) < at.rem) nscale[i] = P.scale[row * P.ss + (at.col + Of<8>::place(i)) / TAD_BLOCK8];
        }
    };
    // the first rows are under way before anything else is done
    if constexpr (V == 8) {
        const unsigned stage = held * (SOURCE_BYTES<S> + (unsigned)sizeof(T));
        ring.start(rows, at.group * STAGES * stage, smem_u32(&bars[at.group][0]), stage, at.in == 0, P.lost);
        if (ring.leader)
            for (int i = 0; i < STAGES; ++i) if (r + i * at.step < P.n_rows) issue(i, r + i * at.step);
        ring.zeros(x_bytes, held * SOURCE_BYTES<S>, at.in, P.group);
        ring.zeros(held * SOURCE_BYTES<S> + dy_bytes, stage, at.in, P.group);
#pragma unroll
        for (int i = 0; i < E / 8; ++i) nscale[i] = 127;
    } else {
        nx.zero();
        ndy.zero();
    }
    fetch(r);
    Pairs<E> w, dws, dbs;
    {
        float f[E];
        load_vector<V, E>(f, P.w, P.w_type, at.col, at.rem, 1.f);
        w.set(f);
    }
    Trade trade;
    if constexpr (BY == BY_CLUSTER) trade.start(P, &ex);
    else if constexpr (V == 8) __syncthreads();
#pragma unroll
    for (int j = 0; j < E / 2; ++j) dws.p[j] = dbs.p[j] = make_float2(0.f, 0.f);
    for (; r < P.n_rows; r += at.step) {
        float xh[E], d[E], xscale[E / 8];
        const float mean = nmean;
        float rstd = nrstd;
        if constexpr (V == 8) {
            const unsigned char *from = ring.row();
            const int c = at.col - at.col0;
            ring.wait();
            if constexpr (PACKED) {
#pragma unroll
                for (int i = 0; i < E / 8; ++i) {
                    uint2 q = *reinterpret_cast<const uint2 *>(from + c + Of<8>::place(i));
                    if (Of<8>::place(i) >= at.rem) q = make_uint2(0, 0);     // (copies end on whole sixteens, eight bytes behind the row at most)
                    float f[8];
                    unpack_eight(q, 1.f, f);
                    xscale[i] = scale_of(nscale[i]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) xh[i * 8 + j] = f[j];
                }
            } else {
                Piece<S, 8> p[E / 8];
                read_row<S, E>(p, reinterpret_cast<const S *>(from) + c);
                elements<S, E>(xh, p);
            }
            Piece<T, 8> p[E / 8];
            read_row<T, E>(p, reinterpret_cast<const T *>(from + held * SOURCE_BYTES<S>) + c);
            elements<T, E>(d, p);
        } else {
            nx.get(xh);
            ndy.get(d);
        }
        fetch(r + at.step);
        if (V == 8 && ring.lost) rstd = __uint_as_float(0x7fffffffu);        // (a row that never came has no result; dw and db: below)
        Pairs<E> h, dp;
        h.set(xh);
        dp.set(d);
        float2 s1 = make_float2(0.f, 0.f), s2 = s1;
#pragma unroll
        for (int j = 0; j < E / 2; ++j) {
            // behind the row xh is zero: zero times an infinite rstd or a NaN mean would reach the sums
            const float2 shift = inside<V>(-mean, j, at.rem);
            // (a packed value times its scale is exact)
            if constexpr (PACKED && V == 8) h.p[j] = __ffma2_rn(h.p[j], make_float2(xscale[j / 4], xscale[j / 4]), shift);
            else h.p[j] = __fadd2_rn(h.p[j], shift);
            h.p[j] = __fmul2_rn(h.p[j], inside<V>(rstd, j, at.rem));
            dws.p[j] = __ffma2_rn(dp.p[j], h.p[j], dws.p[j]);
            dbs.p[j] = __fadd2_rn(dbs.p[j], dp.p[j]);
            const float2 g = __fmul2_rn(dp.p[j], w.p[j]);
            s1 = __fadd2_rn(s1, g);
            s2 = __ffma2_rn(g, h.p[j], s2);
        }
        float s[2] = {s1.x + s1.y, s2.x + s2.y};
        sum.of(s);
        if constexpr (V == 8) {
            // (behind the sum every thread of the group has read the row)
            if (ring.leader && !ring.lost && r + STAGES * at.step < P.n_rows) issue(ring.at, r + STAGES * at.step);
            ring.advance();
        }
        if constexpr (BY == BY_CLUSTER) {
            const float2 *all = trade.with_all(s[0], s[1]);
            s[0] = s[1] = trade.lost ? __uint_as_float(0x7fffffffu) : 0.f;
            for (unsigned b = 0; b < trade.blocks; ++b) { s[0] += all[b].x; s[1] += all[b].y; }
        }
        if (P.dx) {
            const float c1 = -s[0] * P.inv_width, c2 = -s[1] * P.inv_width;
            const float2 rr = make_float2(rstd, rstd), m1 = make_float2(c1, c1), m2 = make_float2(c2, c2);
#pragma unroll
            for (int j = 0; j < E / 2; ++j) dp.p[j] = __fmul2_rn(rr, __ffma2_rn(h.p[j], m2, __ffma2_rn(dp.p[j], w.p[j], m1)));
            dp.get(d);
            store_typed<V, E>(P.dx, P.dx_type, r * P.dxs + at.col, at.rem, d);
        }
    }
    if constexpr (V == 8)
        if (ring.lost) linger();
    if constexpr (BY == BY_CLUSTER) trade.finish();
    if (!P.planes) return;
    if (V == 8 && ring.lost)
#pragma unroll
        for (int j = 0; j < E / 2; ++j) dws.p[j] = dbs.p[j] = make_float2(__uint_as_float(0x7fffffffu), __uint_as_float(0x7fffffffu));
    float dw[E], db[E];
    dws.get(dw);
    dbs.get(db);
    if constexpr (BY == BY_CLUSTER) {
        // one group a block: it owns its columns in the plane of its cluster
        float *plane = P.planes + (size_t)at.row * 2 * P.width + at.col;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (Of<V>::place(e / V) < at.rem) {
                plane[Of<V>::column(e)] = dw[e];
                plane[(size_t)P.width + Of<V>::column(e)] = db[e];
            }
    } else {
        join_groups<V, E>(P, dw, db, V == 8 ? reinterpret_cast<float *>(rows) : join, at.group, at.in, at.col);
    }
}

// rows of any length: the sums and dx of a row by a block, its columns by tad_norm_columns_kernel
template <class S, class T>
__global__ void __launch_bounds__(LARGE)
tad_norm_backward_long_kernel(const Params P)
{
    __shared__ float box[2][2][32];
    tad_wait_previous();
    int turn = 0;
    const T *__restrict__ dys = static_cast<const T *>(P.dy);
    for (int64_t r = blockIdx.x; r < P.n_rows; r += gridDim.x) {
        const T *dy = dys + r * P.dys;
        const float mean = P.mean[r], rstd = P.rstd[r];
        float2 s = make_float2(0.f, 0.f);
        auto at = [&](int c, float &xh) {
            Source<S, 1> p;
            p.load(P, r, c);
            float v[1];
            p.get(v);
            xh = (v[0] - mean) * rstd;
            return to_float(dy[c]) * (P.w ? element(P.w, P.w_type, c) : 1.f);
        };
#pragma unroll 4
        for (int c = threadIdx.x; c < P.width; c += LARGE) {
            float xh;
            const float g = at(c, xh);
            s.x += g;
            s.y += g * xh;
        }
        s.x = warp_sum(s.x);
        s.y = warp_sum(s.y);
        if ((threadIdx.x & 31) == 0) { box[turn][0][threadIdx.x >> 5] = s.x; box[turn][1][threadIdx.x >> 5] = s.y; }
        __syncthreads();
        s.x = warp_sum(box[turn][0][threadIdx.x & 31]);
        s.y = warp_sum(box[turn][1][threadIdx.x & 31]);
        turn ^= 1;
        const float c1 = s.x * P.inv_width, c2 = s.y * P.inv_width;
#pragma unroll 4
        for (int c = threadIdx.x; c < P.width; c += LARGE) {
            float xh;
            const float g = at(c, xh);
            put_element(P.dx, P.dx_type, r * P.dxs + c, rstd * (g - c1 - xh * c2));
        }
    }
}

// planes of dw and db for long rows: a thread owns a column in the rows of its block
template <class S, class T>
__global__ void __launch_bounds__(SMALL)
tad_norm_columns_kernel(const Params P, int64_t rows_each)
{
    tad_wait_previous();
    const int c = blockIdx.x * SMALL + threadIdx.x;
    if (c >= P.width) return;
    const int64_t r0 = blockIdx.y * rows_each, r1 = r0 + rows_each < P.n_rows ? r0 + rows_each : P.n_rows;
    float dw = 0.f, db = 0.f;
#pragma unroll 4
    for (int64_t r = r0; r < r1; ++r) {
        Source<S, 1> p;
        p.load(P, r, c);
        float v[1];
        p.get(v);
        const float d = to_float(static_cast<const T *>(P.dy)[r * P.dys + c]);
        dw += d * ((v[0] - P.mean[r]) * P.rstd[r]);
        db += d;
    }
    float *plane = P.planes + (size_t)blockIdx.y * 2 * P.width;
    plane[c] = dw;
    plane[(size_t)P.width + c] = db;
}

// adds the planes up: 32 columns a block, its 32 warps take every 32nd plane
__global__ void __launch_bounds__(1024)
tad_norm_planes_kernel(const float *__restrict__ planes, int n_planes, int width, void *dw, int dw_type, void *db, int db_type)
{
    __shared__ float part[32][33];
    tad_wait_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float a = 0.f;
    if (c < 2 * (int64_t)width) {
#pragma unroll 4
        for (int p = warp; p < n_planes; p += 32) a += planes[(size_t)p * 2 * width + c];
    }
    part[warp][lane] = a;
    __syncthreads();
    float t = part[lane][warp];            // column `warp` of the block, plane share `lane`
#pragma unroll
    for (int d = 16; d; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
    const int64_t o = (int64_t)blockIdx.x * 32 + warp;
    if (lane != 0 || o >= 2 * (int64_t)width) return;
    if (o < width) { if (dw) put_element(dw, dw_type, o, t); }
    else if (db) put_element(db, db_type, o - width, t);
}

// ---- host ----

// rows of `width` columns by blocks of at most `block` threads, `e` elements a thread
struct Shape { int by, group, cluster; };
Shape shape_of(int64_t width, int block, int e)
{
    Shape s{};
    s.cluster = 1;
    while (s.cluster * (int64_t)block * e < width && s.cluster < MAX_CLUSTER) s.cluster *= 2;
    const int warps = (int)((width + 32 * e - 1) / (32 * e));
    s.by = s.cluster > 1 ? BY_CLUSTER : warps > 1 ? BY_GROUP : BY_WARP;
    s.group = s.by == BY_CLUSTER ? block : s.by == BY_WARP ? 32 : (warps + 1) / 2 * 64;      // (warps in pairs: their sums are read in pairs)
    return s;
}

// the backward pass: blocks of 512 threads or, in clusters that hold the row so, two of 256 an SM, so that two rows are under way there
Shape backward_shape(int64_t width, int e)
{
    const bool halves = width > (int64_t)BACKWARD_BLOCK * e && width <= (int64_t)(BACKWARD_BLOCK / 2) * e * MAX_CLUSTER;
    return shape_of(width, halves ? BACKWARD_BLOCK / 2 : BACKWARD_BLOCK, e);
}

// Planes of partial sums of the backward pass, one a block or cluster: one block an SM, as many groups in it as fit.  The workspace has
// room for those of either number of elements a thread.
int64_t planes_of(int64_t n_rows, int64_t width, int e)
{
    if (width > HELD) return std::max<int64_t>(1, std::min<int64_t>(n_rows, 64));
    const Shape s = backward_shape(width, e);
    const int groups = s.by == BY_CLUSTER ? 1 : BACKWARD_BLOCK / s.group;
    return std::max<int64_t>(1, std::min<int64_t>((n_rows + groups - 1) / groups, SMS * (s.by == BY_CLUSTER ? BACKWARD_BLOCK / s.group : 1) / s.cluster));
}

// Clusters that run at a time: not all SMs of the device have enough neighbours, and one that has to wait for another doubles the time
// (2048 x 16384 bf16 forward 72 us for 49).  The device is asked once for a kernel, its threads and a size of clusters; `known`:
// 64 devices, clusters of 2, 4 and 8.
template <class K>
cudaError_t clusters_of(K kernel, int threads, size_t smem, int cluster, std::atomic<int> (*known)[3], int64_t &most)
{
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::atomic<int> *place = dev >= 0 && dev < 64 ? &known[dev][cluster == 2 ? 0 : cluster == 4 ? 1 : 2] : nullptr;
    int n = place ? place->load(std::memory_order_relaxed) : 0;
    if (!n) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = cluster; cfg.blockDim = threads; cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr = {};
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = cluster; attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr; cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
        if (e != cudaSuccess) return e;
        n = std::max(1, n);
        if (place) place->store(n, std::memory_order_relaxed);
    }
    most = n;
    return cudaSuccess;
}

// dynamic shared memory of a kernel beyond 48 KB, once a device
template <class K>
cudaError_t allow(K kernel, size_t most, std::atomic<bool> (&known)[64])
{
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev >= 0 && dev < 64 && known[dev].load(std::memory_order_relaxed))) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e == cudaSuccess && dev >= 0 && dev < 64) known[dev].store(true, std::memory_order_relaxed);
    return e;
}

constexpr size_t WIDE_ROOM = 220 * 1024;
constexpr int64_t EVEN_BYTES = 96000000;
constexpr int EVEN = 5;

template <class T>
cudaError_t forward(const Params &P, const Shape &s, bool eights, bool keep, cudaStream_t stream)
{
    if (P.width > HELD) return tad_launch(tad_norm_forward_long_kernel<T>, (unsigned)std::min<int64_t>(P.n_rows, 2 * SMS), LARGE, 0, stream, P);
    // Rows that a cluster would hold, by one block, as far as two rows and the weights fit into 220 KB: 13312 columns of fp32, 18432 of 16-bit types
    // (2048 x 16384 bf16 35 us, 2048 x 18440 by clusters 116).  (Of few rows a cluster each is faster: 16 x 16384 4.5 us for 6.6, 200 x 8192 5.4 for 6.4, 300 x 8192
    // 6.9 for 6.7, 1000 x 8192 14 for 10.  Rows up to 4096 in this form: 8192 x 4096 25.3 for 26.5, but 8192 x 2560 22.4 for 20.2, 20000 x 1024 25.6
    // for 17.6, 1000 x 2048 5.6 for 4.5.)
    if (eights && !keep && s.by == BY_CLUSTER && P.width <= WIDE_BLOCK * WIDE_E<T> && P.n_rows >= 2 * SMS) {
        Params W = P;
        W.group = (P.width + 64 * WIDE_E<T> - 1) / (64 * WIDE_E<T>) * 64;
        const size_t held = (size_t)W.group * WIDE_E<T>, vectors = held * 8;
        int groups = std::min(15, WIDE_BLOCK / W.group);           // (named barriers: one a group beside the block's)
        while (groups > 1 && 2 * groups * held * sizeof(T) + vectors > WIDE_ROOM) --groups;
        const int threads = groups * W.group;
        const size_t stage = groups * held * sizeof(T);
        static std::atomic<bool> allowed[2][64];
        if (2 * stage + vectors <= WIDE_ROOM) {
            const bool four = 4 * stage + vectors <= WIDE_ROOM;
            auto kernel = four ? tad_norm_forward_kernel<T, 8, BY_GROUP, false, 4> : tad_norm_forward_kernel<T, 8, BY_GROUP, false, 2>;
            const cudaError_t e = allow(kernel, WIDE_ROOM, allowed[four]);
            if (e != cudaSuccess) return e;
            return tad_launch(kernel, (unsigned)std::min<int64_t>((P.n_rows + groups - 1) / groups, SMS), threads, (four ? 4 : 2) * stage + vectors, stream, W);
        }
    }
    const int threads = s.by == BY_WARP ? FORWARD_BLOCK : s.group, groups = s.by == BY_WARP ? FORWARD_BLOCK / 32 : 1;
    int64_t most = (int64_t)SMS * std::min(32, (eights ? FORWARD_BLOCKS : 2) * FORWARD_BLOCK / threads);
    // Many fp32 rows: memory bounds them, and the SMs get unequal shares of it (8192 x 4096: the first blocks end at 31 us, the last at 46).  Five
    // times the blocks, each with a fifth of the rows and at least three, even that out: 43 us for 48, 32768 x 4096 168 for 193.  16-bit rows
    // are bound by instructions, there the blocks' starts cost more (26.6 -> 31.9), as they do with less to read than L2 holds.
    if (sizeof(T) == 4 && eights && !keep && s.by == BY_GROUP && P.n_rows * P.width * 4 >= EVEN_BYTES && P.n_rows >= 16 * most) most *= EVEN;
    auto kernel = tad_norm_forward_kernel<T, 1, BY_WARP>;
    if (eights) kernel = s.by == BY_WARP ? tad_norm_forward_kernel<T, 8, BY_WARP> : s.by == BY_GROUP ? tad_norm_forward_kernel<T, 8, BY_GROUP> : tad_norm_forward_kernel<T, 8, BY_CLUSTER>;
    else if (s.by != BY_WARP) kernel = s.by == BY_GROUP ? tad_norm_forward_kernel<T, 1, BY_GROUP> : tad_norm_forward_kernel<T, 1, BY_CLUSTER>;
    if constexpr (std::is_same<T, float>::value)
        if (keep) kernel = s.by == BY_WARP ? tad_norm_forward_kernel<T, 8, BY_WARP, true> : s.by == BY_GROUP ? tad_norm_forward_kernel<T, 8, BY_GROUP, true> : tad_norm_forward_kernel<T, 8, BY_CLUSTER, true>;
    const size_t smem = eights ? (size_t)threads * FORWARD_E * sizeof(T) * FORWARD_STAGES<T> : 0;      // (32 KB at most)
    if (s.cluster > 1) {
        static std::atomic<int> known[3][64][3];
        const cudaError_t e = clusters_of(kernel, threads, smem, s.cluster, known[eights + keep], most);
        if (e != cudaSuccess) return e;
    }
    const unsigned blocks = (unsigned)(std::min((P.n_rows + groups - 1) / groups, most) * s.cluster);
    return tad_launch_cluster(kernel, blocks, threads, smem, stream, s.cluster, P);
}

// also says how many planes there are
template <class S, class T>
cudaError_t backward(Params &P, bool eights, int64_t &planes, cudaStream_t stream)
{
    const int e8 = eights ? BACKWARD_E<8> : BACKWARD_E<1>;
    planes = planes_of(P.n_rows, P.width, e8);
    const Shape s = backward_shape(P.width, e8);
    P.group = s.group;
    if (P.width > HELD) {
        cudaError_t e = cudaSuccess;
        if (P.dx) e = tad_launch(tad_norm_backward_long_kernel<S, T>, (unsigned)std::min<int64_t>(P.n_rows, 2 * SMS), LARGE, 0, stream, P);
        if (e == cudaSuccess && P.planes)
            e = tad_launch(tad_norm_columns_kernel<S, T>, dim3((unsigned)((P.width + SMALL - 1) / SMALL), (unsigned)planes), SMALL, 0, stream, P, (P.n_rows + planes - 1) / planes);
        return e;
    }
    auto kernel = tad_norm_backward_kernel<S, T, 1, BY_WARP>;
    if (eights) kernel = s.by == BY_WARP ? tad_norm_backward_kernel<S, T, 8, BY_WARP> : s.by == BY_GROUP ? tad_norm_backward_kernel<S, T, 8, BY_GROUP> : tad_norm_backward_kernel<S, T, 8, BY_CLUSTER>;
    else if (s.by != BY_WARP) kernel = s.by == BY_GROUP ? tad_norm_backward_kernel<S, T, 1, BY_GROUP> : tad_norm_backward_kernel<S, T, 1, BY_CLUSTER>;
    const int threads = s.by == BY_CLUSTER ? s.group : BACKWARD_BLOCK / s.group * s.group;
    size_t smem = 0;
    if (eights) {
        constexpr size_t most = (size_t)BACKWARD_BLOCK * BACKWARD_E<8> * (SOURCE_BYTES<S> + sizeof(T)) * BACKWARD_STAGES<S, T>;
        static_assert(most <= 163840, "rows ahead and the join of the groups fit into shared memory");
        static std::atomic<bool> allowed[3][64];
        const cudaError_t e = allow(kernel, most, allowed[s.by]);
        if (e != cudaSuccess) return e;
        smem = (size_t)threads * BACKWARD_E<8> * (SOURCE_BYTES<S> + sizeof(T)) * BACKWARD_STAGES<S, T>;
    }
    if (s.cluster > 1) {
        static std::atomic<int> known[2][2][64][3];                          // (by the kernel and its threads)
        int64_t most = 0;
        const cudaError_t e = clusters_of(kernel, threads, smem, s.cluster, known[eights][threads == BACKWARD_BLOCK], most);
        if (e != cudaSuccess) return e;
        planes = std::min(planes, most);
    }
    return tad_launch_cluster(kernel, (unsigned)(planes * s.cluster), threads, smem, stream, s.cluster, P);
}

}  // namespace

extern "C" {

void tad_debug_lost_waits(int32_t lost) { lost_waits.store(lost != 0, std::memory_order_relaxed); }

tad_status tad_layernorm_forward(const tad_rows *x, int64_t n_rows, int64_t width, const tad_rows *weight, const tad_rows *bias,
                                 float eps, const tad_rows *y, float *mean, float *rstd, const tad_packed *checkpoint,
                                 void *cuda_stream)
{
    tad_status st;
    if ((st = check_sizes("layernorm_forward", n_rows, width)) || (st = check_rows("layernorm_forward: x", x, n_rows, width)) ||
        (st = check_rows("layernorm_forward: y", y, n_rows, width))) return st;
    if (weight && (st = check_rows("layernorm_forward: weight", weight, 1, width, true))) return st;
    if (bias && (st = check_rows("layernorm_forward: bias", bias, 1, width, true))) return st;
    if (checkpoint && (st = check_packed("layernorm_forward: checkpoint", checkpoint, n_rows, width))) return st;
    if (!(eps >= 0.f)) return bad("layernorm_forward", "eps is negative or NaN");
    if (reinterpret_cast<uintptr_t>(mean) % 4 || reinterpret_cast<uintptr_t>(rstd) % 4) return bad("layernorm_forward", "mean or rstd not aligned");
    if (n_rows == 0) return TAD_OK;
    if (width == 0) {
        if (mean || rstd) return bad("layernorm_forward", "rows of no elements have no mean");
        return TAD_OK;
    }
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    Params P{};
    P.x = x->data; P.xs = x->stride;
    P.y = y->data; P.ys = y->stride; P.y_type = y->type;
    if (weight) { P.w = weight->data; P.w_type = weight->type; }
    if (bias) { P.b = bias->data; P.b_type = bias->type; }
    P.mean = mean; P.rstd = rstd;
    P.n_rows = n_rows; P.width = (int)width; P.eps = eps; P.inv_width = 1.f / (float)width;
    P.lost = lost_waits.load(std::memory_order_relaxed);
    const Shape s = shape_of(width, FORWARD_BLOCK, FORWARD_E);
    P.group = s.group;
    const bool eights = width % 8 == 0 && by_eights(x) && by_eights(y);
    // The checkpoint of fp32 rows in the norm's own pass (8192 x 4096: 51 us for 71); of 16-bit rows, where the pass has no instructions to
    // spare, by the packing kernel, which leaves x in L2 for the next one (16384 x 2048 bf16 43 us either way, 8192 x 4096 44 us for 46).
    const bool keep = checkpoint && x->type == TAD_F32 && eights && width <= HELD;
    if (keep) { P.kq = checkpoint->q; P.kqs = checkpoint->q_stride; P.kscale = checkpoint->scale; P.kss = checkpoint->scale_stride; }
    else if (checkpoint && (st = tad_launch_pack8(x, n_rows, width, checkpoint, stream))) return st;
    cudaError_t e = cudaSuccess;
    TAD_WITH_TYPE(x->type, T, e = forward<T>(P, s, eights, keep, stream));
    return launched("layer norm", e);
}

size_t tad_layernorm_workspace_bytes(int64_t n_rows, int64_t width)
{
    if (n_rows <= 0 || width <= 0 || n_rows >= MAX_ROWS || width >= MAX_WIDTH) return 0;
    return ((size_t)std::max(planes_of(n_rows, width, 16), planes_of(n_rows, width, 8)) * 2 * (size_t)width * 4 + 255) & ~size_t(255);
}

tad_status tad_layernorm_backward(const tad_rows *dy, const tad_rows *x, const tad_packed *checkpoint, int64_t n_rows, int64_t width,
                                  const tad_rows *weight, const float *mean, const float *rstd, const tad_rows *dx,
                                  const tad_rows *dweight, const tad_rows *dbias, void *workspace, size_t workspace_bytes,
                                  void *cuda_stream)
{
    tad_status st;
    if ((st = check_sizes("layernorm_backward", n_rows, width)) || (st = check_rows("layernorm_backward: dy", dy, n_rows, width))) return st;
    if (!x == !checkpoint) return bad("layernorm_backward", "x or a checkpoint of it, one of the two");
    if (x && (st = check_rows("layernorm_backward: x", x, n_rows, width))) return st;
    if (checkpoint && (st = check_packed("layernorm_backward: checkpoint", checkpoint, n_rows, width))) return st;
    if (weight && (st = check_rows("layernorm_backward: weight", weight, 1, width, true))) return st;
    if (dx && (st = check_rows("layernorm_backward: dx", dx, n_rows, width))) return st;
    if (dweight && (st = check_rows("layernorm_backward: dweight", dweight, 1, width, true))) return st;
    if (dbias && (st = check_rows("layernorm_backward: dbias", dbias, 1, width, true))) return st;
    if (width == 0) return TAD_OK;
    if (n_rows > 0 && (!mean || !rstd || reinterpret_cast<uintptr_t>(mean) % 4 || reinterpret_cast<uintptr_t>(rstd) % 4))
        return bad("layernorm_backward", "mean or rstd NULL or not aligned");
    const bool sums = dweight || dbias;
    if (sums && (st = check_room("layernorm_backward", workspace, workspace_bytes, tad_layernorm_workspace_bytes(n_rows, width)))) return st;
    if (!dx && !sums) return TAD_OK;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    int64_t planes = 0;
    if (n_rows > 0) {
        Params P{};
        P.dy = dy->data; P.dys = dy->stride;
        if (x) { P.x = x->data; P.xs = x->stride; }
        else { P.q = checkpoint->q; P.qs = checkpoint->q_stride; P.scale = checkpoint->scale; P.ss = checkpoint->scale_stride; }
        if (weight) { P.w = weight->data; P.w_type = weight->type; }
        if (dx) { P.dx = dx->data; P.dxs = dx->stride; P.dx_type = dx->type; }
        P.mean = const_cast<float *>(mean); P.rstd = const_cast<float *>(rstd);
        P.planes = sums ? static_cast<float *>(workspace) : nullptr;
        P.n_rows = n_rows; P.width = (int)width; P.inv_width = 1.f / (float)width;
        P.lost = lost_waits.load(std::memory_order_relaxed);
        const bool eights = width % 8 == 0 && by_eights(dy) && (!x || by_eights(x)) && (!dx || by_eights(dx));
        TAD_WITH_TYPE(dy->type, T, {
            if (!x) e = backward<Packed8, T>(P, eights, planes, stream);
            else TAD_WITH_TYPE(x->type, S, e = (backward<S, T>(P, eights, planes, stream)));
        });
    }
    if (e == cudaSuccess && sums)
        e = tad_launch(tad_norm_planes_kernel, (unsigned)((2 * width + 31) / 32), 1024, 0, stream, static_cast<const float *>(workspace), (int)planes, (int)width,
                       dweight ? dweight->data : nullptr, dweight ? dweight->type : 0, dbias ? dbias->data : nullptr, dbias ? dbias->type : 0);
    return launched("layer norm backward", e);
}

}  // extern "C"
