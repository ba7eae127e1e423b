// Products of packed matrices (tad_matmul8):  y_ij = sum_k a_ik b_jk,  both operands e4m3 with one power of two for each block of 128 along k.
//
//     y_ij = sum_blocks 2^(sa_i,block) 2^(sb_j,block) sum_{k in block} qa_ik qb_jk
//
// The tensor cores apply the scales themselves (block-scaled MMA, exponent bytes in tensor memory beside the accumulator), so the sum
// over all of k stays in tensor memory and the epilogue reads it once.  The products are exact; the accumulator truncates
// where it aligns summands.
//
// One block an SM, walking over tiles of 128 rows of one operand (p: the lanes of tensor memory) and BN of the other (q).  A warp
// copies 128 x 128 and BN x 128 bytes a stage by TMA (a block of 128 elements is one 128-byte line of the swizzled layout), four warps
// bring the scales of 512 elements at a time from memory into tensor memory, a warp issues the MMAs and eight warps empty the
// accumulator.  Large products run on pairs of blocks (PAIR, clusters of two SMs): a tile of 256 x 256, each block holds 128 rows of p and
// of q and half of the accumulator, and the first block issues the MMAs of both.  What bounds those is L2: at the full rate of the
// tensor cores single tiles of 128 x 256 would read 27 TB/s from it.  Measured, bf16 out: 8192 x 4096 x 4096 99 us (2.8 PFLOP/s; 112 - 120 us
// in a row without a pause, where the power limit sets the clock), 8192 x 8192 x 8192 361 - 374 us (3.0 - 2.9); with one MMA of four left the
// loop takes 64 of the 99 us, so the tensor cores and their clock are what remains.
#include <cuda.h>

#include <atomic>

#include "rows.cuh"

namespace {

using namespace tadr;

constexpr int BM = 128, KB = 128;                 // rows of p in a tile; bytes of a row in a stage (a block of the scales)
constexpr int SF_BLOCKS = 4, SF_BUFFERS = 8;      // blocks whose scales are one word of tensor memory (a chunk); chunks in tensor memory
constexpr int EPI_WARPS = 8, SF_WARPS = 4, NT = 512;
// registers: 512 threads start with 128 each; the last two warpgroups go down to 56, the two that empty the accumulator up to 200
constexpr int REG_EPI = 200, REG_REST = 56;
constexpr long long WAIT_LIMIT = 1ll << 32;       // clocks after which a wait gives up (about two seconds; a tile takes 0.1 s at most)
constexpr int STAGE_ROOM = 163840;                // shared memory of the stages
constexpr int TURN_PITCH = 33, TURN_ROOM = EPI_WARPS * 32 * TURN_PITCH * 4;      // 32 x 32 results of a warp on their way to rows off 32-byte boundaries

// ---- PTX ----
__device__ __forceinline__ unsigned smem_u32(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(unsigned bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
// `bar` of block `rank` of the cluster
__device__ __forceinline__ unsigned at_block(unsigned bar, unsigned rank)
{
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(bar), "r"(rank));
    return r;
}
// Relaxed: what the blocks of a pair tell each other so lies in tensor memory (written or read by completed instructions, in front of the fence
// for them).  A release would wait for every earlier access of the thread: 2 us for the scales of a chunk, whose MMAs take 1.
__device__ __forceinline__ void mbar_arrive_far(unsigned bar) { asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void mbar_arrive(unsigned bar) { asm volatile("{ .reg .b64 t; mbarrier.arrive.shared::cta.b64 t, [%0]; }" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void mbar_expect(unsigned bar, unsigned bytes) { asm volatile("{ .reg .b64 t; mbarrier.arrive.expect_tx.shared::cta.b64 t, [%0], %1; }" ::"r"(bar), "r"(bytes) : "memory"); }
__device__ __forceinline__ bool mbar_try(unsigned bar, unsigned parity)
{
    unsigned ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// (by whole warps) false: this wait ran out, or another one of the block did
__device__ __forceinline__ bool mbar_wait(unsigned bar, unsigned parity, volatile int *failed)
{
    if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
    const long long start = clock64();
    do {
        if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
        if (__any_sync(0xffffffffu, *failed != 0)) return false;
    } while (!__any_sync(0xffffffffu, clock64() - start > WAIT_LIMIT));
    *failed = 1;
    return false;
}
// the same after a failure: only to let what is in flight arrive
__device__ __forceinline__ void mbar_drain(unsigned bar, unsigned parity)
{
    const long long start = clock64();
    while (!__all_sync(0xffffffffu, mbar_try(bar, parity)) && !__any_sync(0xffffffffu, clock64() - start > WAIT_LIMIT)) { }
}
// about a millisecond: a thousand times what a copy takes
__device__ __forceinline__ void linger()
{
    const long long start = clock64();
    while (clock64() - start < (1ll << 21)) { }
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tma_load(unsigned to, const CUtensorMap *map, int x, int y, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// the same by either block of a pair, counted at a barrier of the first one
__device__ __forceinline__ void tma_load_pair(unsigned to, const CUtensorMap *map, int x, int y, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// by a whole warp with uniform operands, one elected lane issues
template <bool PAIR>
__device__ __forceinline__ void mma_scaled(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned sfa, unsigned sfb, unsigned acc)
{
    if (PAIR)
        asm volatile("{ .reg .pred p, q; elect.sync _|q, 0xffffffff; setp.ne.u32 p, %6, 0;\n"
                     "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p; }" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(acc) : "memory");
    else
        asm volatile("{ .reg .pred p, q; elect.sync _|q, 0xffffffff; setp.ne.u32 p, %6, 0;\n"
                     "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p; }" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(acc) : "memory");
}
// arrives at the barrier (PAIR: of both blocks) when the MMAs so far are done
template <bool PAIR>
__device__ __forceinline__ void mma_commit(unsigned bar)
{
    if (PAIR)
        asm volatile("{ .reg .pred q; .reg .b16 m; mov.b16 m, 3; elect.sync _|q, 0xffffffff; @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m; }" ::"r"(bar) : "memory");
    else
        asm volatile("{ .reg .pred q; elect.sync _|q, 0xffffffff; @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld32(unsigned addr, float (&v)[32])
{
    unsigned r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st4(unsigned addr, const unsigned (&r)[4])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
// shared-memory matrix descriptor: K-major, 128-byte swizzle, eight rows of 128 bytes per repeat
__device__ __forceinline__ unsigned long long make_desc(unsigned addr)
{
    return (unsigned long long)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

struct Product {
    const uint8_t *sp, *sq;                       // scales of both operands
    int64_t sps, sqs;
    void *y;                                      // or the planes of a split product
    int64_t yp, yq;                               // element strides of y along p and q: one of them is 1
    int64_t plane;                                // elements of a plane, 0 without a split
    int type, vec;                                // vec: stores of 32 bytes along q
    int np, nq, blocks, each, split;              // sizes, blocks of k, blocks of a share of k, shares
    unsigned tiles_p, tiles_q, tiles;
    int lost;                                     // a wait for a tile's operands counts as run out (tests)
};

template <int BN, bool PAIR> struct Config {
    static constexpr int ROWS_Q = PAIR ? BN / 2 : BN;                     // rows of q that a block copies
    static constexpr int STAGE = (BM + ROWS_Q) * KB, STAGES = STAGE_ROOM / STAGE < 8 ? STAGE_ROOM / STAGE : 8;
    static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + TURN_ROOM;
    static constexpr int SF_COLS = 16;                                    // columns of a buffer of scales: four of p, up to eight of q
};

// tiles of one share of k in groups of sixteen along p, so that the blocks that run together share operand lines in L2
__device__ __forceinline__ void tile_at(const Product &P, unsigned t, int &p0, int &q0, int &share, int bm, int bn)
{
    const unsigned per = P.tiles_p * P.tiles_q;
    share = (int)(t / per);
    t -= (unsigned)share * per;
    const unsigned group = 16u * P.tiles_q, g = t / group, first = g * 16u, size = min(16u, P.tiles_p - first), in = t - g * group;
    p0 = (int)(first + in % size) * bm;
    q0 = (int)(in / size) * bn;
}

// four bytes of results
template <class T> __device__ __forceinline__ unsigned word_of(const float *v);
template <> __device__ __forceinline__ unsigned word_of<float>(const float *v) { return __float_as_uint(v[0]); }
template <> __device__ __forceinline__ unsigned word_of<__nv_bfloat16>(const float *v) { const __nv_bfloat162 h = __floats2bfloat162_rn(v[0], v[1]); return *reinterpret_cast<const unsigned *>(&h); }
template <> __device__ __forceinline__ unsigned word_of<__half>(const float *v) { const __half2 h = __floats2half2_rn(v[0], v[1]); return *reinterpret_cast<const unsigned *>(&h); }

// all threads of the block or pair
template <bool PAIR>
__device__ __forceinline__ void block_sync()
{
    if (PAIR) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else __syncthreads();
}

template <int BN, bool PAIR>
__global__ void __launch_bounds__(NT, 1)
tad_product8_kernel(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q, const Product P)
{
    using C = Config<BN, PAIR>;
    constexpr int S = C::STAGES, TILE_P = PAIR ? 2 * BM : BM;
    extern __shared__ unsigned char smem_raw[];
    __shared__ unsigned long long bars[2 * S + 2 * SF_BUFFERS + 3];
    __shared__ unsigned tmem_base, spread[2][BM + (BN < 128 ? 128 : BN)];
    __shared__ volatile int failed;
    const unsigned smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const unsigned full = smem_u32(&bars[0]), empty = full + 8 * S, sf_full = empty + 8 * S, sf_empty = sf_full + 8 * SF_BUFFERS, acc_full = sf_empty + 8 * SF_BUFFERS, acc_empty = acc_full + 8, mma_end = acc_empty + 8;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const unsigned rank = PAIR ? blockIdx.x & 1 : 0;                      // in the pair; the first block issues the MMAs
    const unsigned walker = PAIR ? blockIdx.x >> 1 : blockIdx.x, walkers = PAIR ? gridDim.x >> 1 : gridDim.x;
    if (warp == EPI_WARPS) {
        if (lane == 0) {
            failed = 0;
            for (int i = 0; i < S; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
            for (int i = 0; i < SF_BUFFERS; ++i) { mbar_init(sf_full + 8 * i, PAIR ? 2 * SF_WARPS : SF_WARPS); mbar_init(sf_empty + 8 * i, 1); }
            mbar_init(acc_full, 1);
            mbar_init(mma_end, 1);
            mbar_init(acc_empty, PAIR ? 2 * EPI_WARPS : EPI_WARPS);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_base)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_base)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    fence_before();
    block_sync<PAIR>();
    fence_after();
    tad_wait_previous();
    const unsigned tmem = __shfl_sync(0xffffffffu, tmem_base, 0);
    constexpr unsigned SF = 256;                                          // first column of the scales
    bool ok = true;

    if (warp >= EPI_WARPS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REG_REST));
    if (warp > EPI_WARPS + SF_WARPS + 1) {
        // (the rest of the last warpgroup)
    } else if (warp == EPI_WARPS + SF_WARPS) {
        // ---- copies ----
        int at = 0;
        unsigned long long issued = 0;
        for (unsigned t = walker; t < P.tiles && ok; t += walkers) {
            int p0, q0, share;
            tile_at(P, t, p0, q0, share, TILE_P, BN);
            const int b1 = min(P.blocks, (share + 1) * P.each);
            for (int b = share * P.each; b < b1; ++b) {
                const int turn = (int)(issued / S);
                if (turn > 0 && !(ok = mbar_wait(empty + 8 * at, (turn - 1) & 1, &failed))) break;
                if (lane == 0) {
                    const unsigned to = smem0 + at * C::STAGE, bar = full + 8 * at;
                    if (PAIR) {                        // the first block's barrier counts the bytes of both
                        if (rank == 0) mbar_expect(bar, 2 * C::STAGE);
                        const unsigned far = at_block(bar, 0), own = at_block(to, rank);
                        tma_load_pair(own, &map_p, b * KB, p0 + (int)rank * BM, far);
                        tma_load_pair(own + BM * KB, &map_q, b * KB, q0 + (int)rank * C::ROWS_Q, far);
                    } else {
                        mbar_expect(bar, C::STAGE);
                        tma_load(to, &map_p, b * KB, p0, bar);
                        tma_load(to + BM * KB, &map_q, b * KB, q0, bar);
                    }
                }
                __syncwarp();
                ++issued;
                if (++at == S) at = 0;
            }
        }
        // copies of a block that gave up still write its shared memory (of a pair: the first block's barriers know, of those that both have issued)
        if (!ok && rank != 0) linger();
        if (!ok && rank == 0)
            for (unsigned long long i = issued > S ? issued - S : 0; i < issued; ++i) mbar_drain(full + 8 * (unsigned)(i % S), (unsigned)(i / S) & 1);
    } else if (warp == EPI_WARPS + SF_WARPS + 1) {
        // ---- products ----
        const unsigned base = ((unsigned)BN >> 3 << 17) | (1u << 23) | ((unsigned)(TILE_P >> 4) << 24);
        int at = 0, phase = 0, sf = 0, sf_phase = 0, n = 0;
        for (unsigned t = walker; t < P.tiles && ok && rank == 0; t += walkers, ++n) {
            int p0, q0, share;
            tile_at(P, t, p0, q0, share, TILE_P, BN);
            const int b0 = share * P.each, b1 = min(P.blocks, b0 + P.each);
            if (n > 0) ok = mbar_wait(acc_empty, (n - 1) & 1, &failed);
            for (int b = b0; b < b1 && ok; ++b) {
                const int in = (b - b0) % SF_BLOCKS;
                if (in == 0) ok = mbar_wait(sf_full + 8 * sf, sf_phase, &failed);
                ok = ok && mbar_wait(full + 8 * at, phase, &failed);
                if (!ok) break;
                fence_after();
                const unsigned st = smem0 + at * C::STAGE;
                const unsigned long long da = make_desc(st), db = make_desc(st + BM * KB);
                const unsigned idesc = base | ((unsigned)in << 4) | ((unsigned)in << 29);
                const unsigned sfa = tmem + SF + sf * C::SF_COLS;
#pragma unroll
                for (int kk = 0; kk < KB / 32; ++kk) mma_scaled<PAIR>(tmem, da + 2 * kk, db + 2 * kk, idesc, sfa, sfa + 4, b > b0 || kk > 0);
                mma_commit<PAIR>(empty + 8 * at);
                if (++at == S) { at = 0; phase ^= 1; }
                if (in == SF_BLOCKS - 1 || b + 1 == b1) {
                    mma_commit<PAIR>(sf_empty + 8 * sf);
                    if (++sf == SF_BUFFERS) { sf = 0; sf_phase ^= 1; }
                }
            }
            if (P.lost) { failed = 1; ok = false; }               // (not in the loop over k: 512 x 4096 x 4096 13.5 us for 11.9)
            if (ok) mma_commit<PAIR>(acc_full);
        }
        // MMAs of a block that gave up still read its shared memory: all are done when this commit arrives.  It has a barrier of its own, which
        // nobody else waits at: at acc_full it would pass the part of a sum that there is for the sum.  (And copies that are under way behind
        // those that were waited for get the time to land.)
        if (!ok && rank == 0) {
            mma_commit<PAIR>(mma_end);
            mbar_drain(mma_end, 0);
            linger();
        }
    } else if (warp >= EPI_WARPS) {
        // ---- scales: lane l of every quarter of tensor memory holds rows l, 32 + l, ... in columns 0, 1, ..., the scale of one block a byte.
        // A thread loads the words of one row of p and one or two of q, DEEP chunks ahead, and they are spread to the lanes through shared
        // memory (loaded by every warp for itself they are 32 rows an instruction).  Eight buffers: the chain from memory to tensor memory is
        // longer than the MMAs of a chunk, but never theirs to wait for ----
        constexpr int ROWS = BM + (BN < 128 ? 128 : BN), OWN = ROWS / (SF_WARPS * 32), DEEP = 4;
        const int quad = warp & 3, thread = threadIdx.x - EPI_WARPS * 32;
        unsigned at_t = walker;                                    // the next chunk to be loaded
        int p0 = 0, q0 = 0, b = 0, b1 = 0;
        auto tile = [&] {
            int share;
            if (at_t >= P.tiles) return;
            tile_at(P, at_t, p0, q0, share, TILE_P, BN);
            b = share * P.each;
            b1 = min(P.blocks, b + P.each);
        };
        unsigned mine[DEEP][OWN];
        bool there[DEEP];
        auto load = [&](unsigned (&w)[OWN]) {                      // false: there is no further chunk
            if (at_t >= P.tiles) return false;
#pragma unroll
            for (int g = 0; g < OWN; ++g) {
                const int in = thread + (g - 1) * 128;             // among the rows of q (g > 0)
                const int64_t row = g == 0 ? p0 + (int)rank * BM + thread : q0 + in;
                w[g] = 0x7f7f7f7fu;
                if (row < (g == 0 ? P.np : P.nq) && (g == 0 || in < BN))
                    w[g] = *reinterpret_cast<const unsigned *>(g == 0 ? P.sp + row * P.sps + b : P.sq + row * P.sqs + b);
            }
            b += SF_BLOCKS;
            if (b >= b1) { at_t += walkers; tile(); }
            return true;
        };
        tile();
#pragma unroll
        for (int d = 0; d < DEEP; ++d) there[d] = load(mine[d]);
        for (int turn = 0; there[0]; ) {
#pragma unroll
            for (int d = 0; d < DEEP; ++d) {
                if (!there[d]) { there[0] = false; break; }
                unsigned *room = spread[d & 1];
#pragma unroll
                for (int g = 0; g < OWN; ++g) room[g * 128 + thread] = mine[d][g];
                there[d] = load(mine[d]);
                // (the room of two turns ago has been read by all four warps: they have met at the barrier of the turn between)
                asm volatile("bar.sync 1, 128;" ::: "memory");
                unsigned w[OWN][4];
#pragma unroll
                for (int g = 0; g < OWN; ++g)
#pragma unroll
                    for (int c = 0; c < 4; ++c) w[g][c] = room[g * 128 + c * 32 + lane];
                const int sf = turn % SF_BUFFERS;
                if (turn >= SF_BUFFERS && ok) ok = mbar_wait(sf_empty + 8 * sf, (turn / SF_BUFFERS - 1) & 1, &failed);
                ++turn;
                if (!ok) continue;                                 // (all four warps stay in step at the barrier)
                fence_after();
                const unsigned to = tmem + ((unsigned)(quad * 32) << 16) + SF + sf * C::SF_COLS;
#pragma unroll
                for (int g = 0; g < OWN; ++g) tmem_st4(to + 4 * g, w[g]);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                fence_before();
                __syncwarp();
                if (lane == 0) { if (PAIR) mbar_arrive_far(at_block(sf_full + 8 * sf, 0)); else mbar_arrive(sf_full + 8 * sf); }
            }
        }
    } else {
        // ---- results: a warp empties a quarter of the lanes in half of the columns, all of them into registers before the first is stored, so
        // that the next tile's MMAs wait for that alone (there is room for one accumulator of 256 columns beside the scales) ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REG_EPI));
        constexpr int HALF = BN >= 64 ? BN / 2 : 32;                                       // columns that a warp reads
        const int quad = warp & 3, half = BN >= 64 ? warp >> 2 : 0;
        const bool idle = BN < 64 && warp >= 4;
        int n = 0;
        for (unsigned t = walker; t < P.tiles; t += walkers, ++n) {
            int p0, q0, share;
            tile_at(P, t, p0, q0, share, TILE_P, BN);
            ok = ok && mbar_wait(acc_full, n & 1, &failed);
            fence_after();
            float v[HALF];
            if (ok && !idle) {
                const unsigned from = tmem + ((unsigned)(quad * 32) << 16) + half * HALF;
#pragma unroll
                for (int c = 0; c < HALF; c += 32) tmem_ld32(from + c, *reinterpret_cast<float (*)[32]>(&v[c]));
                tmem_wait_ld();
            } else {
#pragma unroll
                for (int j = 0; j < HALF; ++j) v[j] = __uint_as_float(0x7fffffffu);         // a wait ran out: nothing that looks like a result
            }
            fence_before();
            __syncwarp();
            if (lane == 0) { if (PAIR) mbar_arrive_far(at_block(acc_empty, 0)); else mbar_arrive(acc_empty); }
            const int p = p0 + (int)rank * BM + quad * 32 + lane;
            const int live = p < P.np && !idle ? min(HALF, P.nq - q0 - half * HALF) : 0;       // columns of this thread
            const int64_t o = P.plane * share + p * P.yp + (int64_t)(q0 + half * HALF) * P.yq;
            auto put = [&](auto *out) {
                using T = typename std::remove_pointer<decltype(out)>::type;
                T *to = out + o;
                if (P.vec && __all_sync(0xffffffffu, live == HALF)) {
#pragma unroll
                    for (int j = 0; j < HALF; j += 32 / (int)sizeof(T)) {                     // 32 bytes: whole sectors
                        unsigned w[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k] = word_of<T>(&v[j + k * (4 / (int)sizeof(T))]);
                        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to + j), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
                    }
                } else if (P.yq == 1) {
                    // a row of 32 results by one store of the warp: by each lane for its row they are 32 sectors a store (1500 x 1333 x 1100 fp32
                    // 28 us for 15)
                    float *turn = reinterpret_cast<float *>(smem_raw + (smem0 - smem_u32(smem_raw)) + S * C::STAGE) + warp * (32 * TURN_PITCH);
                    const int rows = idle ? 0 : min(32, P.np - (p - lane)), columns = min(HALF, P.nq - q0 - half * HALF);
#pragma unroll
                    for (int c = 0; c < HALF; c += 32) {
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 32; ++j) turn[lane * TURN_PITCH + j] = v[c + j];
                        __syncwarp();
                        if (c + lane < columns) {
                            T *at = out + (o - lane * P.yp) + c + lane;
#pragma unroll 8
                            for (int r = 0; r < rows; ++r) at[r * P.yp] = from_float<T>(turn[r * TURN_PITCH + lane]);
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < HALF; ++j) if (j < live) to[j * P.yq] = from_float<T>(v[j]);
                }
            };
            if (P.type == TAD_F32) put(static_cast<float *>(P.y));
            else if (P.type == TAD_BF16) put(static_cast<__nv_bfloat16 *>(P.y));
            else put(static_cast<__half *>(P.y));
        }
    }
    fence_before();
    block_sync<PAIR>();
    fence_after();
    if (warp == EPI_WARPS) {
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// ---- few rows ----

// Up to four rows on one side and little work: bound by its launch and one round of loads.  A warp takes two rows of the other operand and
// sixteen elements of k a lane and step, the few rows come from the first-level cache.  Five instructions an element, of one row, make it
// slower than the tensor cores from some 20 million multiply-adds on; us, these / those: 1 x 256 x 256 2.0 / 4.4, 4 x 1000 x 1000 4.3 / 5.8,
// 1 x 4096 x 4096 6.3 / 7.5, 2 x 4096 x 4096 8.9 / 7.5, 1 x 65536 x 512 15 / 11, 1 x 16384 x 8192 35 / 27.
constexpr int FEW = 4, FEW_ROWS = 2;
constexpr int64_t FEW_WORK = int64_t(20) << 20;

struct Few {
    const uint8_t *q, *s, *fq, *fs;                // the many rows, the few rows
    int64_t qs, ss, fqs, fss, y_many, y_few;       // strides
    void *y;
    int type, many, few, k;
};

// A lane's sixteen elements lie in one block on either side.  Their products are summed as the codes stand for them (448^2 16 at most) and the
// scales applied to the sum, as two powers of two of the same size: 2^120 times an element is beyond fp32, and so is its product with an element
// of the other side, where that side's scale brings it back.  (The first factor loses digits of a sum only where the second
// makes it less than the smallest fp32 number; where it gives an infinity, so does the second.)
template <int F>
__global__ void __launch_bounds__(128)
tad_product8_few_kernel(const Few P)
{
    tad_wait_previous();
    const int lane = threadIdx.x & 31;
    const int64_t r0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 5)) * FEW_ROWS;
    if (r0 >= P.many) return;
    float acc[FEW_ROWS][F];
#pragma unroll
    for (int i = 0; i < FEW_ROWS; ++i)
#pragma unroll
        for (int f = 0; f < F; ++f) acc[i][f] = 0.f;
#pragma unroll F == 1 ? 4 : 2
    for (int k = lane * 16; k < P.k; k += 512) {
        // (rows are a multiple of 16 bytes: the load is inside; what lies behind k counts as zero)
        const int left = P.k - k;
        uint4 w[FEW_ROWS];
        unsigned ws[FEW_ROWS], xs[F];
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i) {
            const int64_t r = min(r0 + i, (int64_t)P.many - 1);
            w[i] = *reinterpret_cast<const uint4 *>(P.q + r * P.qs + k);
            ws[i] = (unsigned)P.s[r * P.ss + k / TAD_BLOCK8] << 23;
        }
        float x[F][16];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int g = min(f, P.few - 1);
            const uint4 u = *reinterpret_cast<const uint4 *>(P.fq + g * P.fqs + k);
            xs[f] = (unsigned)P.fs[g * P.fss + k / TAD_BLOCK8] << 23;
            float lo[8], hi[8];
            unpack_eight(make_uint2(u.x, u.y), 1.f, lo);
            unpack_eight(make_uint2(u.z, u.w), 1.f, hi);
#pragma unroll
            for (int j = 0; j < 8; ++j) { x[f][j] = lo[j]; x[f][8 + j] = hi[j]; }
            if (left < 16)
#pragma unroll
                for (int j = 0; j < 16; ++j) if (j >= left) x[f][j] = 0.f;
            if (xs[f] == 255u << 23) x[f][0] = __uint_as_float(0x7fffffffu);           // (a block whose scale stands for NaN)
        }
#pragma unroll
        for (int i = 0; i < FEW_ROWS; ++i) {
            float v[16], lo[8], hi[8];
            unpack_eight(make_uint2(w[i].x, w[i].y), 1.f, lo);
            unpack_eight(make_uint2(w[i].z, w[i].w), 1.f, hi);
#pragma unroll
            for (int j = 0; j < 8; ++j) { v[j] = lo[j]; v[8 + j] = hi[j]; }
            if (left < 16)
#pragma unroll
                for (int j = 0; j < 16; ++j) if (j >= left) v[j] = 0.f;
            if (ws[i] == 255u << 23) v[0] = __uint_as_float(0x7fffffffu);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                float2 d = make_float2(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < 16; j += 2) d = __ffma2_rn(make_float2(v[j], v[j + 1]), make_float2(x[f][j], x[f][j + 1]), d);
                // (the sum of two exponent bytes has nine bits; a byte of 0 is a factor 0 here instead of 2^-127, in results below 2^-230)
                const unsigned both = ws[i] + xs[f], half = both >> 1 & 0x7f800000u;
                acc[i][f] = fmaf((d.x + d.y) * __uint_as_float(half), __uint_as_float(both - half), acc[i][f]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < FEW_ROWS; ++i)
#pragma unroll
        for (int f = 0; f < F; ++f) {
            float a = acc[i][f];
#pragma unroll
            for (int d = 16; d; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
            if (lane == 0 && r0 + i < P.many && f < P.few) put_element(P.y, P.type, (r0 + i) * P.y_many + f * P.y_few, a);
        }
}

// y from the planes of a split product
__global__ void __launch_bounds__(256)
tad_product8_planes_kernel(const float *__restrict__ planes, int n_planes, int64_t m, int n, void *y, int64_t ys, int type)
{
    tad_wait_previous();
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= m * n) return;
    float a = 0.f;
#pragma unroll 4
    for (int p = 0; p < n_planes; ++p) a += planes[p * m * n + e];
    const int64_t i = e / n;
    put_element(y, type, i * ys + (e - i * n), a);
}

__global__ void __launch_bounds__(256)
tad_product8_zero_kernel(int64_t m, int n, void *y, int64_t ys, int type)
{
    tad_wait_previous();
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= m * n) return;
    put_element(y, type, e / n * ys + e % n, 0.f);
}

// ---- host ----

// how a product is run: the longer side is p where the other one fits into one tile
struct Way {
    bool few, p_is_b, pair;
    int bn, split, each, blocks;
    int64_t tiles_p, tiles_q;
};
Way way_of(int64_t m, int64_t n, int64_t k)
{
    Way w{};
    const int64_t s = std::min(m, n);
    w.blocks = (int)blocks_of(k);
    w.few = s <= FEW && s * std::max(m, n) * k <= FEW_WORK;
    w.split = 1;
    w.p_is_b = s <= 128 && n > m;
    if (w.few) return w;
    const int64_t np = w.p_is_b ? n : m, nq = w.p_is_b ? m : n;
    w.tiles_p = (np + BM - 1) / BM;
    auto tiles = [&](int bn) { return w.tiles_p * ((nq + bn - 1) / bn); };
    if (nq <= 32) w.bn = 32;
    else if (nq <= 64) w.bn = 64;
    else {
        const double t256 = (double)((tiles(256) + SMS - 1) / SMS), t128 = 0.55 * (double)((tiles(128) + SMS - 1) / SMS);
        w.bn = nq > 128 && t256 <= t128 ? 256 : 128;
    }
    // pairs where they have work for all SMs
    const int64_t pairs = ((np + 2 * BM - 1) / (2 * BM)) * ((nq + 255) / 256);
    w.pair = nq > 128 && pairs >= SMS / 2;
    if (w.pair) { w.bn = 256; w.tiles_p = (np + 2 * BM - 1) / (2 * BM); }
    w.tiles_q = (nq + w.bn - 1) / w.bn;
    // fewer tiles than SMs: k in shares of whole words of scales
    const int64_t t = w.tiles_p * w.tiles_q;
    int64_t split = t < SMS && !w.pair ? std::min<int64_t>(SMS / t, (w.blocks + 2 * SF_BLOCKS - 1) / (2 * SF_BLOCKS)) : 1;
    split = std::max<int64_t>(1, split);
    w.each = (int)((w.blocks + split - 1) / split);
    w.each = (w.each + SF_BLOCKS - 1) / SF_BLOCKS * SF_BLOCKS;
    w.split = (w.blocks + w.each - 1) / w.each;
    return w;
}

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled()
{
    static std::atomic<void *> known{nullptr};
    void *f = known.load(std::memory_order_relaxed);
    if (!f) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) { cudaGetLastError(); return nullptr; }
        known.store(f, std::memory_order_relaxed);
    }
    return reinterpret_cast<EncodeTiled>(f);
}

bool map_of(CUtensorMap *map, const tad_packed *m, int64_t rows, int64_t k, int box_rows)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t size[2] = {(cuuint64_t)k, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)m->q_stride};
    const cuuint32_t box[2] = {KB, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, m->q, size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, bool PAIR>
cudaError_t launch_product(const CUtensorMap &mp, const CUtensorMap &mq, const Product &P, cudaStream_t stream)
{
    static std::atomic<bool> allowed[64];
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !allowed[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(tad_product8_kernel<BN, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Config<BN, PAIR>::SMEM);
        if (e != cudaSuccess) return e;
        // the warpgroups' register shares must fit into what the block is launched with
        cudaFuncAttributes at;
        e = cudaFuncGetAttributes(&at, tad_product8_kernel<BN, PAIR>);
        if (e != cudaSuccess) return e;
        if (at.numRegs * NT < EPI_WARPS * 32 * REG_EPI + (NT - EPI_WARPS * 32) * REG_REST) return cudaErrorInvalidConfiguration;
        if (dev >= 0 && dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
    }
    if (PAIR) return tad_launch_cluster(tad_product8_kernel<BN, PAIR>, 2 * std::min(P.tiles, (unsigned)SMS / 2), NT, Config<BN, PAIR>::SMEM, stream, 2, mp, mq, P);
    return tad_launch(tad_product8_kernel<BN, PAIR>, std::min(P.tiles, (unsigned)SMS), NT, Config<BN, PAIR>::SMEM, stream, mp, mq, P);
}

}  // namespace

extern "C" {

size_t tad_matmul8_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (m <= 0 || n <= 0 || k <= 0 || m >= MAX_ROWS || n >= MAX_ROWS || k >= MAX_WIDTH) return 0;
    const Way w = way_of(m, n, k);
    return w.split > 1 ? ((size_t)w.split * (size_t)m * (size_t)n * 4 + 255) & ~size_t(255) : 0;
}

tad_status tad_matmul8(const tad_packed *a, const tad_packed *b, int64_t m, int64_t n, int64_t k, const tad_rows *y,
                       void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    tad_status st;
    if ((st = check_sizes("matmul8", m, k)) || (st = check_sizes("matmul8", n, k)) || (st = check_packed("matmul8: a", a, m, k)) ||
        (st = check_packed("matmul8: b", b, n, k)) || (st = check_rows("matmul8: y", y, m, n))) return st;
    if (m == 0 || n == 0) return TAD_OK;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    const int64_t elements = m * n;
    if (elements >= (int64_t(1) << 38)) return refuse(TAD_ERR_UNSUPPORTED, "matmul8", "2^38 outputs and more");
    if (k == 0) return launched("product", tad_launch(tad_product8_zero_kernel, (unsigned)((elements + 255) / 256), 256, 0, stream, m, (int)n, y->data, y->stride, (int)y->type));
    const Way w = way_of(m, n, k);
    if ((st = check_room("matmul8", workspace, workspace_bytes, tad_matmul8_workspace_bytes(m, n, k)))) return st;
    cudaError_t e = cudaSuccess;
    if (w.few) {
        const bool b_many = n > m;
        const tad_packed *many = b_many ? b : a, *few = b_many ? a : b;
        Few P{};
        P.q = many->q; P.qs = many->q_stride; P.s = many->scale; P.ss = many->scale_stride;
        P.fq = few->q; P.fqs = few->q_stride; P.fs = few->scale; P.fss = few->scale_stride;
        P.y = y->data; P.type = y->type; P.y_many = b_many ? 1 : y->stride; P.y_few = b_many ? y->stride : 1;
        P.many = (int)(b_many ? n : m); P.few = (int)(b_many ? m : n); P.k = (int)k;
        const unsigned grid = (unsigned)((P.many + 4 * FEW_ROWS - 1) / (4 * FEW_ROWS));
        e = tad_launch(P.few == 1 ? tad_product8_few_kernel<1> : P.few == 2 ? tad_product8_few_kernel<2> : tad_product8_few_kernel<FEW>, grid, 128, 0, stream, P);
        return launched("product", e);
    }
    const tad_packed *p = w.p_is_b ? b : a, *q = w.p_is_b ? a : b;
    Product P{};
    P.np = (int)(w.p_is_b ? n : m); P.nq = (int)(w.p_is_b ? m : n);
    P.sp = p->scale; P.sps = p->scale_stride; P.sq = q->scale; P.sqs = q->scale_stride;
    P.blocks = w.blocks; P.each = w.each; P.split = w.split;
    P.tiles_p = (unsigned)w.tiles_p; P.tiles_q = (unsigned)w.tiles_q;
    const int64_t tiles = w.tiles_p * w.tiles_q * w.split;
    if (tiles >= MAX_ROWS) return refuse(TAD_ERR_UNSUPPORTED, "matmul8", "too many tiles");
    P.tiles = (unsigned)tiles;
    P.lost = lost_waits.load(std::memory_order_relaxed);
    int64_t stride = y->stride;
    P.y = y->data; P.type = y->type;
    if (w.split > 1) { P.y = workspace; P.type = TAD_F32; P.plane = elements; stride = n; }
    P.yp = w.p_is_b ? 1 : stride; P.yq = w.p_is_b ? stride : 1;
    P.vec = !w.p_is_b && reinterpret_cast<uintptr_t>(P.y) % 32 == 0 && stride * (int64_t)type_size(P.type) % 32 == 0 && P.plane % 8 == 0;
    CUtensorMap mp, mq;
    if (!map_of(&mp, p, P.np, k, BM) || !map_of(&mq, q, P.nq, k, w.pair ? w.bn / 2 : w.bn)) return refuse(TAD_ERR_CUDA, "matmul8", "no tensor map for this matrix (or no driver)");
    e = w.pair ? launch_product<256, true>(mp, mq, P, stream) : w.bn == 256 ? launch_product<256, false>(mp, mq, P, stream) : w.bn == 128 ? launch_product<128, false>(mp, mq, P, stream) :
        w.bn == 64 ? launch_product<64, false>(mp, mq, P, stream) : launch_product<32, false>(mp, mq, P, stream);
    if (e == cudaSuccess && w.split > 1)
        e = tad_launch(tad_product8_planes_kernel, (unsigned)((elements + 255) / 256), 256, 0, stream, static_cast<const float *>(workspace), w.split, m, (int)n, y->data, y->stride, (int)y->type);
    return launched("product", e);
}

}  // extern "C"
