// Matrices in 8 bits (tad_pack8, tad_unpack8, tad_repack8): blocks of 128 elements of a row in e4m3 with a power of two as scale.
//
//     k = min { j >= -126 : max |x| <= 448 2^j },   q = e4m3(x 2^-k),   x ~ q 2^k
//
// The scale is a power of two, so it is one byte, the division is exact, q depends on x alone (no rounding of a scale that
// another order of operations would make different) and the tensor cores can apply it to a block's products.
// All three move bytes and are bound by memory.
#include "rows.cuh"

namespace {

using namespace tadr;

constexpr int NT = 256, ROWS = 4;          // threads of a block; rows that a thread has under way

// Sixteen threads own a block of 128, eight elements each.  A thread block covers CB = 2^cb_log blocks of a row (16 or, in narrow
// matrices, the whole row) and ROWS x 16 / CB rows.
struct Cover {
    int64_t row0;            // first row of this thread, the next ones are `step` rows on
    int step, blk;           // its block of 128 in the row
    int col;                 // first of its eight elements
    __device__ __forceinline__ Cover(int cb_log, unsigned chunks)
    {
        const unsigned group = blockIdx.x / chunks, chunk = blockIdx.x - group * chunks;
        const int b = threadIdx.x >> 4;
        step = 16 >> cb_log;
        row0 = (int64_t)group * (ROWS * step) + (b >> cb_log);
        blk = (int)(chunk << cb_log) + (b & ((1 << cb_log) - 1));
        col = blk * TAD_BLOCK8 + (threadIdx.x & 15) * 8;
    }
};

// eight elements from c on, zeros behind the row; VEC: 16-byte loads where all eight exist
template <class T, bool VEC>
__device__ __forceinline__ void load_eight(float (&v)[8], const T *__restrict__ row, int c, int width)
{
    if (VEC && c + 8 <= width) {
        Piece<T, 8> p;
        p.load(row + c);
        p.get(v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < width ? to_float(row[c + j]) : 0.f;
    }
}

__device__ __forceinline__ float max_of_block(float a)
{
#pragma unroll
    for (int d = 8; d; d >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
    return a;
}

template <class T, bool VEC>
__global__ void __launch_bounds__(NT)
tad_pack8_kernel(const T *__restrict__ x, int64_t xs, int64_t n_rows, int width, int n_blocks, int cb_log, unsigned chunks,
                 uint8_t *__restrict__ q, int64_t qs, uint8_t *__restrict__ scale, int64_t ss)
{
    tad_wait_previous();
    const Cover at(cb_log, chunks);
    float v[ROWS][8];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = at.row0 + i * at.step;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        if (r < n_rows && at.col < width) load_eight<T, VEC>(v[i], x + r * xs, at.col, width);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = at.row0 + i * at.step;
        float a = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) a = fmaxf(a, finite_abs(v[i][j]));
        const unsigned s = scale_byte(max_of_block(a));
        if (r >= n_rows || at.col >= width) continue;
        const uint2 p = pack_eight(v[i], inverse_scale(s));
        uint8_t *to = q + r * qs + at.col;
        if (at.col + 8 <= width) *reinterpret_cast<uint2 *>(to) = p;
        else for (int j = 0; j < width - at.col; ++j) to[j] = (uint8_t)((j < 4 ? p.x : p.y) >> (8 * (j & 3)));
        if ((threadIdx.x & 15) == 0) scale[r * ss + at.blk] = (uint8_t)s;
    }
}

template <class T, bool VEC>
__global__ void __launch_bounds__(NT)
tad_unpack8_kernel(const uint8_t *__restrict__ q, int64_t qs, const uint8_t *__restrict__ scale, int64_t ss, int64_t n_rows, int width,
                   int cb_log, unsigned chunks, T *__restrict__ x, int64_t xs)
{
    tad_wait_previous();
    const Cover at(cb_log, chunks);
    uint2 p[ROWS];
    unsigned s[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = at.row0 + i * at.step;
        if (r < n_rows && at.col < width) {
            // (rows of q are a multiple of 16 long: all eight bytes exist)
            p[i] = *reinterpret_cast<const uint2 *>(q + r * qs + at.col);
            s[i] = scale[r * ss + at.blk];
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = at.row0 + i * at.step;
        if (r >= n_rows || at.col >= width) continue;
        float v[8];
        unpack_eight(p[i], scale_of(s[i]), v);
        T *to = x + r * xs + at.col;
        if (VEC && at.col + 8 <= width) {
            Piece<T, 8> o;
            o.set(v);
            o.store(to);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) if (at.col + j < width) to[j] = from_float<T>(v[j]);
        }
    }
}

// The transpose, 128 x 128 elements a thread block: warp w holds rows 16 w .. 16 w + 15 and lane g columns 4 g .. 4 g + 3 in
// registers (a row is one coalesced line of 128 bytes), the largest value of a column is found over the warps through shared
// memory, and the packed columns pass through shared memory as 16-byte units, unit u of column c at place u ^ ((c / 4) mod 8), so that
// neither side has bank conflicts and each row of the output gets its 128 bytes at once.
__global__ void __launch_bounds__(NT)
tad_repack8_kernel(const uint8_t *__restrict__ q, int64_t qs, const uint8_t *__restrict__ scale, int64_t ss, int64_t n_rows, int width,
                   unsigned tiles_c, uint8_t *__restrict__ out, int64_t os, uint8_t *__restrict__ oscale, int64_t oss)
{
    __shared__ float most[8][128];
    __shared__ uint4 tile[128 * 8];
    tad_wait_previous();
    const unsigned tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    const int warp = threadIdx.x >> 5, g = threadIdx.x & 31;
    const int64_t r0 = (int64_t)tr * 128;
    const int c0 = (int)tc * 128, c = c0 + 4 * g;
    unsigned w[16], s[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t r = r0 + warp * 16 + i;
        const bool live = r < n_rows && c < width;
        w[i] = live ? *reinterpret_cast<const unsigned *>(q + r * qs + c) : 0u;
        s[i] = live ? scale[r * ss + tc] : 127u;
    }
    float v[16][4], a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float f = scale_of(s[i]);
        const float2 lo = from_e4m3x2(w[i] & 0xffffu), hi = from_e4m3x2(w[i] >> 16);
        v[i][0] = lo.x * f; v[i][1] = lo.y * f; v[i][2] = hi.x * f; v[i][3] = hi.y * f;
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = fmaxf(a[j], finite_abs(v[i][j]));
    }
    *reinterpret_cast<float4 *>(&most[warp][4 * g]) = make_float4(a[0], a[1], a[2], a[3]);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float4 m = *reinterpret_cast<const float4 *>(&most[i][4 * g]);
        a[0] = fmaxf(a[0], m.x); a[1] = fmaxf(a[1], m.y); a[2] = fmaxf(a[2], m.z); a[3] = fmaxf(a[3], m.w);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const unsigned b = scale_byte(a[j]);
        const float inv = inverse_scale(b);
        unsigned u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            u[i] = to_e4m3x2(v[4 * i][j] * inv, v[4 * i + 1][j] * inv) | (to_e4m3x2(v[4 * i + 2][j] * inv, v[4 * i + 3][j] * inv) << 16);
        tile[(4 * g + j) * 8 + (warp ^ (g & 7))] = make_uint4(u[0], u[1], u[2], u[3]);
        if (warp == 0 && c + j < width) oscale[(int64_t)(c + j) * oss + tr] = (uint8_t)b;
    }
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
            for (int j = 0; j < 16 && at + j < n_rows; ++j) to[j] = (uint8_t)(words[j >> 2] >> (8 * (j & 3)));
        }
    }
}

struct Launch { unsigned blocks, chunks; int cb_log; };
Launch cover(int64_t n_rows, int64_t n_blocks)
{
    Launch l{0, 0, 0};
    while (l.cb_log < 4 && (int64_t(1) << l.cb_log) < n_blocks) ++l.cb_log;
    l.chunks = (unsigned)((n_blocks + (1 << l.cb_log) - 1) >> l.cb_log);
    const int64_t rows = ROWS * (16 >> l.cb_log);
    l.blocks = (unsigned)((n_rows + rows - 1) / rows * l.chunks);
    return l;
}

}  // namespace

// also called by the layer norm for a checkpoint that its own pass cannot write
tad_status tad_launch_pack8(const tad_rows *x, int64_t n_rows, int64_t width, const tad_packed *out, cudaStream_t stream)
{
    const Launch l = cover(n_rows, tadr::blocks_of(width));
    cudaError_t e = cudaSuccess;
    const bool vec = by_eights(x);
    TAD_WITH_TYPE(x->type, T,
        auto kernel = vec ? tad_pack8_kernel<T, true> : tad_pack8_kernel<T, false>;
        e = tad_launch(kernel, l.blocks, NT, 0, stream, static_cast<const T *>(x->data), x->stride, n_rows, (int)width,
                       (int)tadr::blocks_of(width), l.cb_log, l.chunks, out->q, out->q_stride, out->scale, out->scale_stride));
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
    const Launch l = cover(n_rows, blocks_of(width));
    cudaError_t e = cudaSuccess;
    const bool vec = by_eights(x);
    TAD_WITH_TYPE(x->type, T,
        auto kernel = vec ? tad_unpack8_kernel<T, true> : tad_unpack8_kernel<T, false>;
        e = tad_launch(kernel, l.blocks, NT, 0, (cudaStream_t)cuda_stream, in->q, in->q_stride, in->scale, in->scale_stride, n_rows, (int)width,
                       l.cb_log, l.chunks, static_cast<T *>(x->data), x->stride));
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
    if (tiles >= MAX_ROWS) { tad::set_error("repack8: too many tiles"); return TAD_ERR_UNSUPPORTED; }
    return launched("repack", tad_launch(tad_repack8_kernel, (unsigned)tiles, NT, 0, (cudaStream_t)cuda_stream, in->q, in->q_stride, in->scale,
                                         in->scale_stride, n_rows, (int)width, tiles_c, out->q, out->q_stride, out->scale, out->scale_stride));
}

}  // extern "C"
