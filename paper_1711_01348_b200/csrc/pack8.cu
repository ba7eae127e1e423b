// Matrices in 8 bits (tad_pack8, tad_unpack8, tad_repack8): blocks of 128 elements of a row in e4m3 with a power of two as scale.
//
//     k = min { j >= -126 : max |x| <= 448 2^j },   q = e4m3(x 2^-k),   x ~ q 2^k
//
// The scale is a power of two, so it is one byte, the division is exact, q depends on x alone (no rounding of a scale that
// another order of operations would make different) and the tensor cores can apply it to a block's products.
// All three move bytes and are bound by memory.  Measured, 16384 x 8192 bf16: packed in 60 us, unpacked in 62 (6.5 TB/s), turned in 79
// (3.4 TB/s: about ten instructions an element, half of the issue slots).
#include "rows.cuh"

namespace {

using namespace tadr;

constexpr int NT = 256, ROWS = 4;          // threads of a block; rows that a thread has under way

// A block of 128 belongs to 2^own neighbouring threads: to pack, eight (sixteen elements each); to unpack, sixteen, because a thread's store
// is one piece of 16 bytes then (two of them, 32 bytes apart in a warp: 81 % of the memory rate for 97 %).  A thread block covers 2^cb
// blocks of a row (all that its threads own or, in narrow matrices, the whole row), and ROWS times as many rows as that leaves it
// threads for.
struct Cover {
    int64_t row0;            // first row of this thread, the next ones are `step` rows on
    int step, blk, in;       // its block of 128 in the row, its place among the block's threads
    __device__ __forceinline__ Cover(int own, int cb, unsigned chunks)
    {
        const unsigned group = blockIdx.x / chunks, chunk = blockIdx.x - group * chunks;
        const int b = threadIdx.x >> own;
        step = (NT >> own) >> cb;
        row0 = (int64_t)group * (ROWS * step) + (b >> cb);
        blk = (int)(chunk << cb) + (b & ((1 << cb) - 1));
        in = threadIdx.x & ((1 << own) - 1);
    }
};
constexpr int OWN_PACK = 3, OWN_UNPACK = 4;

template <class T>
__global__ void __launch_bounds__(NT)
tad_pack8_kernel(const T *__restrict__ x, int64_t xs, int64_t n_rows, int width, int cb, unsigned chunks,
                 uint8_t *__restrict__ q, int64_t qs, uint8_t *__restrict__ scale, int64_t ss)
{
    tad_wait_previous();
    const Cover at(OWN_PACK, cb, chunks);
    const int col = at.blk * TAD_BLOCK8 + at.in * 16;
    Sixteen<T> v[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = at.row0 + i * at.step;
        v[i].zero();
        if (r < n_rows && col < width) v[i].load(x + r * xs, col, width);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = at.row0 + i * at.step;
        unsigned s;
        const uint4 u = v[i].pack(s);
        if (r >= n_rows || col >= width) continue;
        uint8_t *to = q + r * qs + col;
        if (col + 16 <= width) *reinterpret_cast<uint4 *>(to) = u;
        else {
            const unsigned words[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 16; ++j) if (col + j < width) to[j] = (uint8_t)(words[j >> 2] >> (8 * (j & 3)));
        }
        if (at.in == 0) scale[r * ss + at.blk] = (uint8_t)s;
    }
}

template <class T>
__global__ void __launch_bounds__(NT)
tad_unpack8_kernel(const uint8_t *__restrict__ q, int64_t qs, const uint8_t *__restrict__ scale, int64_t ss, int64_t n_rows, int width,
                   int cb, unsigned chunks, T *__restrict__ x, int64_t xs)
{
    tad_wait_previous();
    const Cover at(OWN_UNPACK, cb, chunks);
    const int col = at.blk * TAD_BLOCK8 + at.in * 8;
    uint2 p[ROWS];
    unsigned s[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = at.row0 + i * at.step;
        if (r < n_rows && col < width) {
            // (rows of q are a multiple of 16 long: all eight bytes exist)
            p[i] = *reinterpret_cast<const uint2 *>(q + r * qs + col);
            s[i] = scale[r * ss + at.blk];
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = at.row0 + i * at.step;
        if (r >= n_rows || col >= width) continue;
        float v[8];
        unpack_eight(p[i], scale_of(s[i]), v);
        T *to = x + r * xs + col;
        if (col + 8 <= width) {
            Piece<T, 8> o;
            o.set(v);
            o.store(to);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) if (col + j < width) to[j] = from_float<T>(v[j]);
        }
    }
}

// Rows of x off 16-byte boundaries: a warp a row and ODD blocks of 128, four elements of each a lane, 32 apart, so that every access is
// the lane's pointer and a constant.
constexpr int ODD = 4;

template <class T>
__global__ void __launch_bounds__(NT)
tad_pack8_odd_kernel(const T *__restrict__ x, int64_t xs, int64_t n_rows, int width, unsigned chunks,
                     uint8_t *__restrict__ q, int64_t qs, uint8_t *__restrict__ scale, int64_t ss)
{
    tad_wait_previous();
    const int64_t unit = (int64_t)blockIdx.x * (NT / 32) + (threadIdx.x >> 5), r = unit / chunks;
    if (r >= n_rows) return;
    const int lane = threadIdx.x & 31, c = (int)(unit - r * chunks) * (ODD * TAD_BLOCK8) + lane, rem = width - c;
    const T *__restrict__ from = x + r * xs + c;
    uint8_t *__restrict__ to = q + r * qs + c;
    T raw[4 * ODD];
#pragma unroll
    for (int i = 0; i < 4 * ODD; ++i) {
        raw[i] = from_float<T>(0.f);
        if (32 * i < rem) raw[i] = from[32 * i];
    }
#pragma unroll
    for (int k = 0; k < ODD; ++k) {
        float v[4], a = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[j] = to_float(raw[4 * k + j]); a = fmaxf(a, finite_abs(v[j])); }
#pragma unroll
        for (int d = 16; d; d >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
        const unsigned s = scale_byte(a);
        const float inv = inverse_scale(s);
        const unsigned lo = to_e4m3x2(no_infinity(v[0]) * inv, no_infinity(v[1]) * inv), hi = to_e4m3x2(no_infinity(v[2]) * inv, no_infinity(v[3]) * inv);
#pragma unroll
        for (int j = 0; j < 4; ++j) if (32 * (4 * k + j) < rem) to[32 * (4 * k + j)] = (uint8_t)((j < 2 ? lo : hi) >> (8 * (j & 1)));
        if (lane == 0 && 128 * k < rem) scale[r * ss + c / TAD_BLOCK8 + k] = (uint8_t)s;
    }
}

template <class T>
__global__ void __launch_bounds__(NT)
tad_unpack8_odd_kernel(const uint8_t *__restrict__ q, int64_t qs, const uint8_t *__restrict__ scale, int64_t ss, int64_t n_rows, int width,
                       unsigned chunks, T *__restrict__ x, int64_t xs)
{
    tad_wait_previous();
    const int64_t unit = (int64_t)blockIdx.x * (NT / 32) + (threadIdx.x >> 5), r = unit / chunks;
    if (r >= n_rows) return;
    const int lane = threadIdx.x & 31, c = (int)(unit - r * chunks) * (ODD * TAD_BLOCK8) + lane, rem = width - c;
    const uint8_t *__restrict__ from = q + r * qs + c;
    T *__restrict__ to = x + r * xs + c;
    uint8_t p[4 * ODD], s[ODD];
#pragma unroll
    for (int k = 0; k < ODD; ++k) {
        s[k] = 127;
        if (128 * k < rem + lane) s[k] = scale[r * ss + c / TAD_BLOCK8 + k];         // (the block exists: its first column is c - lane + 128 k)
    }
#pragma unroll
    for (int i = 0; i < 4 * ODD; ++i) {
        p[i] = 0;
        if (32 * i < rem) p[i] = from[32 * i];
    }
#pragma unroll
    for (int k = 0; k < ODD; ++k) {
        const float f = scale_of(s[k]);
        const float2 lo = from_e4m3x2(p[4 * k] | (unsigned)p[4 * k + 1] << 8), hi = from_e4m3x2(p[4 * k + 2] | (unsigned)p[4 * k + 3] << 8);
        const float v[4] = {lo.x * f, lo.y * f, hi.x * f, hi.y * f};
#pragma unroll
        for (int j = 0; j < 4; ++j) if (32 * (4 * k + j) < rem) to[32 * (4 * k + j)] = from_float<T>(v[j]);
    }
}

// The transpose, 128 x 128 elements a thread block: warp w holds rows 16 w .. 16 w + 15 and lane g columns 4 g .. 4 g + 3 in
// registers (a row is one coalesced line of 128 bytes), turned at once into words of four rows of a column.  The largest value of a
// column is found over the warps through shared memory, and the packed columns pass through shared memory as 16-byte units,
// unit u of column c at place u ^ ((c / 4) mod 8), so that neither side has bank conflicts and each row of the output gets its 128
// bytes at once.  Values are formed twice from the bytes: kept, they take 64 registers more.
__global__ void __launch_bounds__(NT, 3)
tad_repack8_kernel(const uint8_t *__restrict__ q, int64_t qs, const uint8_t *__restrict__ scale, int64_t ss, int64_t n_rows, int width,
                   unsigned tiles_c, uint8_t *__restrict__ out, int64_t os, uint8_t *__restrict__ oscale, int64_t oss)
{
    __shared__ __align__(16) float most[8][128], row_scale[128];
    __shared__ uint4 tile[128 * 8];
    tad_wait_previous();
    const unsigned tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    const int warp = threadIdx.x >> 5, g = threadIdx.x & 31;
    const int64_t r0 = (int64_t)tr * 128;
    const int c0 = (int)tc * 128, c = c0 + 4 * g;
    if (threadIdx.x < 128) row_scale[threadIdx.x] = r0 + threadIdx.x < n_rows ? scale_or_infinity(scale[(r0 + threadIdx.x) * ss + tc]) : 1.f;
    unsigned t[4][4];                      // [column][four rows]
    {
        unsigned w[16];
        const uint8_t *from = q + (r0 + warp * 16) * qs + c;
        const int rows = c < width ? (int)min((int64_t)16, n_rows - r0 - warp * 16) : 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            w[i] = 0;
            if (i < rows) w[i] = *reinterpret_cast<const unsigned *>(from);
            from += qs;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned lo0 = __byte_perm(w[4 * k], w[4 * k + 1], 0x5140), hi0 = __byte_perm(w[4 * k], w[4 * k + 1], 0x7362);
            const unsigned lo1 = __byte_perm(w[4 * k + 2], w[4 * k + 3], 0x5140), hi1 = __byte_perm(w[4 * k + 2], w[4 * k + 3], 0x7362);
            t[0][k] = __byte_perm(lo0, lo1, 0x5410); t[1][k] = __byte_perm(lo0, lo1, 0x7632);
            t[2][k] = __byte_perm(hi0, hi1, 0x5410); t[3][k] = __byte_perm(hi0, hi1, 0x7632);
        }
    }
    __syncthreads();
    // rows 4 k .. 4 k + 3 of a column, with their scales
    auto values = [&](unsigned word, const float4 &f, float2 &x, float2 &y) {
        x = __fmul2_rn(from_e4m3x2(word & 0xffffu), make_float2(f.x, f.y));
        y = __fmul2_rn(from_e4m3x2(word >> 16), make_float2(f.z, f.w));
    };
    float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float4 f = *reinterpret_cast<const float4 *>(&row_scale[warp * 16 + 4 * k]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float2 x, y;
            values(t[j][k], f, x, y);
            a[j] = fmaxf(fmaxf(a[j], fmaxf(fabsf(x.x), fabsf(x.y))), fmaxf(fabsf(y.x), fabsf(y.y)));
        }
    }
    // a value can be infinite where its scale is 2^120 or more, or stands for NaN; such values do not count and become NaN
    const bool rare = __syncthreads_or(isinf(a[0]) || isinf(a[1]) || isinf(a[2]) || isinf(a[3]));
    if (rare) {
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 f = *reinterpret_cast<const float4 *>(&row_scale[warp * 16 + 4 * k]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float2 x, y;
                values(t[j][k], f, x, y);
                a[j] = fmaxf(fmaxf(a[j], fmaxf(finite_abs(x.x), finite_abs(x.y))), fmaxf(finite_abs(y.x), finite_abs(y.y)));
            }
        }
    }
    *reinterpret_cast<float4 *>(&most[warp][4 * g]) = make_float4(a[0], a[1], a[2], a[3]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float4 m = *reinterpret_cast<const float4 *>(&most[i][4 * g]);
        a[0] = fmaxf(a[0], m.x); a[1] = fmaxf(a[1], m.y); a[2] = fmaxf(a[2], m.z); a[3] = fmaxf(a[3], m.w);
    }
    float inv[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const unsigned b = scale_byte(a[j]);
        inv[j] = inverse_scale(b);
        if (warp == 0 && c + j < width) oscale[(int64_t)(c + j) * oss + tr] = (uint8_t)b;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float4 f = *reinterpret_cast<const float4 *>(&row_scale[warp * 16 + 4 * k]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float2 x, y;
            values(t[j][k], f, x, y);
            if (rare) { x.x = no_infinity(x.x); x.y = no_infinity(x.y); y.x = no_infinity(y.x); y.y = no_infinity(y.y); }
            const float2 n = make_float2(inv[j], inv[j]);
            x = __fmul2_rn(x, n);
            y = __fmul2_rn(y, n);
            t[j][k] = to_e4m3x2(x.x, x.y) | (to_e4m3x2(y.x, y.y) << 16);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) tile[(4 * g + j) * 8 + (warp ^ (g & 7))] = make_uint4(t[j][0], t[j][1], t[j][2], t[j][3]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 32 + (threadIdx.x >> 3), u = threadIdx.x & 7;
        if (c0 + row >= width) continue;
        const uint4 p = tile[row * 8 + (u ^ ((row >> 2) & 7))];
        const int64_t at = r0 + u * 16;
        uint8_t *to = out + (int64_t)(c0 + row) * os + at;
        if (at + 16 <= n_rows) *reinterpret_cast<uint4 *>(to) = p;
        else {
            const unsigned words[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
            for (int j = 0; j < 16; ++j) if (at + j < n_rows) to[j] = (uint8_t)(words[j >> 2] >> (8 * (j & 3)));
        }
    }
}

struct Launch { unsigned blocks, chunks; int cb; };
// false: more blocks than a launch has (of matrices beyond any memory)
bool cover(int64_t n_rows, int64_t n_blocks, int own, Launch &l)
{
    l = Launch{0, 0, 0};
    while ((NT >> own >> l.cb) > 1 && (int64_t(1) << l.cb) < n_blocks) ++l.cb;
    l.chunks = (unsigned)((n_blocks + (1 << l.cb) - 1) >> l.cb);
    const int64_t rows = ROWS * (NT >> own >> l.cb);
    const int64_t blocks = (n_rows + rows - 1) / rows * l.chunks;
    l.blocks = (unsigned)blocks;
    return blocks < MAX_ROWS;
}

// a warp a row and ODD blocks of 128
bool odd_cover(int64_t n_rows, int64_t width, unsigned &blocks, unsigned &chunks)
{
    const int64_t c = (width + ODD * TAD_BLOCK8 - 1) / (ODD * TAD_BLOCK8), b = (n_rows * c + NT / 32 - 1) / (NT / 32);
    blocks = (unsigned)b;
    chunks = (unsigned)c;
    return b < MAX_ROWS;
}

}  // namespace

// also called by the layer norm for a checkpoint that its own pass cannot write
tad_status tad_launch_pack8(const tad_rows *x, int64_t n_rows, int64_t width, const tad_packed *out, cudaStream_t stream)
{
    cudaError_t e = cudaSuccess;
    if (by_eights(x)) {
        Launch l;
        if (!cover(n_rows, tadr::blocks_of(width), OWN_PACK, l)) return refuse(TAD_ERR_UNSUPPORTED, "pack8", "too many blocks");
        TAD_WITH_TYPE(x->type, T,
            e = tad_launch(tad_pack8_kernel<T>, l.blocks, NT, 0, stream, static_cast<const T *>(x->data), x->stride, n_rows, (int)width, l.cb, l.chunks, out->q,
                           out->q_stride, out->scale, out->scale_stride));
    } else {
        unsigned blocks = 0, chunks = 0;
        if (!odd_cover(n_rows, width, blocks, chunks)) return refuse(TAD_ERR_UNSUPPORTED, "pack8", "too many blocks");
        TAD_WITH_TYPE(x->type, T,
            e = tad_launch(tad_pack8_odd_kernel<T>, blocks, NT, 0, stream, static_cast<const T *>(x->data), x->stride, n_rows, (int)width, chunks, out->q,
                           out->q_stride, out->scale, out->scale_stride));
    }
    return launched("pack", e);
}

extern "C" {

tad_status tad_pack8(const tad_rows *x, int64_t n_rows, int64_t width, const tad_packed *out, void *cuda_stream)
{
    tad_status st;
    if ((st = check_sizes("pack8", n_rows, width)) || (st = check_rows("pack8: x", x, n_rows, width)) || (st = check_packed("pack8: out", out, n_rows, width))) return st;
    if (n_rows == 0 || width == 0) return TAD_OK;
    return tad_launch_pack8(x, n_rows, width, out, (cudaStream_t)cuda_stream);
}

tad_status tad_unpack8(const tad_packed *in, int64_t n_rows, int64_t width, const tad_rows *x, void *cuda_stream)
{
    tad_status st;
    if ((st = check_sizes("unpack8", n_rows, width)) || (st = check_packed("unpack8: in", in, n_rows, width)) || (st = check_rows("unpack8: x", x, n_rows, width))) return st;
    if (n_rows == 0 || width == 0) return TAD_OK;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaSuccess;
    if (by_eights(x)) {
        Launch l;
        if (!cover(n_rows, blocks_of(width), OWN_UNPACK, l)) return refuse(TAD_ERR_UNSUPPORTED, "unpack8", "too many blocks");
        TAD_WITH_TYPE(x->type, T,
            e = tad_launch(tad_unpack8_kernel<T>, l.blocks, NT, 0, stream, in->q, in->q_stride, in->scale, in->scale_stride, n_rows, (int)width, l.cb, l.chunks,
                           static_cast<T *>(x->data), x->stride));
    } else {
        unsigned blocks = 0, chunks = 0;
        if (!odd_cover(n_rows, width, blocks, chunks)) return refuse(TAD_ERR_UNSUPPORTED, "unpack8", "too many blocks");
        TAD_WITH_TYPE(x->type, T,
            e = tad_launch(tad_unpack8_odd_kernel<T>, blocks, NT, 0, stream, in->q, in->q_stride, in->scale, in->scale_stride, n_rows, (int)width, chunks,
                           static_cast<T *>(x->data), x->stride));
    }
    return launched("unpack", e);
}

tad_status tad_repack8(const tad_packed *in, int64_t n_rows, int64_t width, const tad_packed *out, void *cuda_stream)
{
    tad_status st;
    if ((st = check_sizes("repack8", n_rows, width)) || (st = check_sizes("repack8", width, n_rows)) ||
        (st = check_packed("repack8: in", in, n_rows, width)) || (st = check_packed("repack8: out", out, width, n_rows))) return st;
    if (n_rows == 0 || width == 0) return TAD_OK;
    const unsigned tiles_c = (unsigned)blocks_of(width);
    const int64_t tiles = blocks_of(n_rows) * tiles_c;
    if (tiles >= MAX_ROWS) return refuse(TAD_ERR_UNSUPPORTED, "repack8", "too many tiles");
    return launched("repack", tad_launch(tad_repack8_kernel, (unsigned)tiles, NT, 0, (cudaStream_t)cuda_stream, in->q, in->q_stride, in->scale,
                                         in->scale_stride, n_rows, (int)width, tiles_c, out->q, out->q_stride, out->scale, out->scale_stride));
}

}  // extern "C"
