// Layer norm over rows (tad_layernorm_forward, tad_layernorm_backward).
//
//     mean = sum x / D,  rstd = (sum (x - mean)^2 / D + eps)^(-1/2),  xh = (x - mean) rstd,  y = xh w + b
//     g = dy w,  dx = rstd (g - sum g / D - xh sum (g xh) / D),  dw = sum_rows dy xh,  db = sum_rows dy
//
// Both passes read every element once and are bound by memory.  A row is held in registers, sixteen elements a thread, by a warp
// (up to 512 columns) or a block, which walks over the rows that are its share with the next row's loads under way; the
// variance is the mean of the squared deviations of those registers (no difference of large sums).  Weights stay in registers
// over all rows.  The backward pass keeps its share of dw and db there too and writes them once, as a plane of partial
// sums; a second kernel adds the planes up in a fixed order.  Rows longer than a block holds are read twice or three times.
#include "rows.cuh"

tad_status tad_launch_pack8(const tad_rows *x, int64_t n_rows, int64_t width, const tad_packed *out, cudaStream_t stream);

namespace {

using namespace tadr;

constexpr int E = 16;                      // elements of a row in a thread's registers
constexpr int WARP_WIDTH = 32 * E;         // rows that a warp holds
constexpr int SMALL = 256, LARGE = 1024;   // threads of a block: with and without the weights in registers
constexpr int HELD = LARGE * E;            // longest row that a block holds

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
    float eps, inv_width;
};

// sums of two values over the warp or, `warps` > 1, over the block: the same bits in every thread
__device__ __forceinline__ float2 warp_sum(float2 v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) { v.x += __shfl_xor_sync(0xffffffffu, v.x, d); v.y += __shfl_xor_sync(0xffffffffu, v.y, d); }
    return v;
}
// `box`: 2 x 32 places used in turn, so that one barrier a sum is enough
struct Sum {
    float2 (*box)[32];
    int turn;
    template <bool WARP>
    __device__ __forceinline__ float2 of(float2 v)
    {
        v = warp_sum(v);
        if (WARP) return v;
        const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) box[turn][threadIdx.x >> 5] = v;
        __syncthreads();
        v = lane < warps ? box[turn][lane] : make_float2(0.f, 0.f);
        turn ^= 1;
        return warp_sum(v);
    }
};

// V elements of the vector `p` from column c on (zero behind the row)
template <int V>
__device__ __forceinline__ void load_vector(float (&v)[V], const void *p, int type, int c, int width, float none)
{
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = !p ? none : c + j < width ? element(p, type, c + j) : 0.f;
}

template <int V>
__device__ __forceinline__ void store_typed(void *base, int type, int64_t at, const float (&v)[V])
{
    if (type == TAD_F32) { Piece<float, V> o; o.set(v); o.store(static_cast<float *>(base) + at); }
    else if (type == TAD_BF16) { Piece<__nv_bfloat16, V> o; o.set(v); o.store(static_cast<__nv_bfloat16 *>(base) + at); }
    else { Piece<__half, V> o; o.set(v); o.store(static_cast<__half *>(base) + at); }
}

// ---- forward ----

// V = 8: width and all row starts are whole pieces of eight.  HOLD: the weights stay in registers.  KEEP: x goes into 8 bits
// beside the pass (V = 8: sixteen neighbouring threads hold a block of 128).
template <class T, int V, bool WARP, bool HOLD, bool KEEP>
__global__ void __launch_bounds__(HOLD ? SMALL : LARGE, HOLD ? 3 : 1)
tad_norm_forward_kernel(const Params P)
{
    constexpr int NV = E / V;
    __shared__ float2 box[2][32];
    tad_wait_previous();
    Sum sum{box, 0};
    const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, span = WARP ? 32 : blockDim.x;
    const int64_t step = WARP ? (int64_t)gridDim.x * (SMALL / 32) : gridDim.x;
    int64_t r = WARP ? (int64_t)blockIdx.x * (SMALL / 32) + (threadIdx.x >> 5) : blockIdx.x;
    const T *__restrict__ x = static_cast<const T *>(P.x);
    const int width = P.width;
    float w[HOLD ? NV : 1][V], b[HOLD ? NV : 1][V];
    if constexpr (HOLD) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * span + tid) * V;
            load_vector<V>(w[i], P.w, P.w_type, c, width, 1.f);
            load_vector<V>(b[i], P.b, P.b_type, c, width, 0.f);
        }
    }
    Piece<T, V> next[NV];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * span + tid) * V;
            next[i].zero();
            if (row < P.n_rows && c < width) next[i].load(x + row * P.xs + c);
        }
    };
    fetch(r);
    for (; r < P.n_rows; r += step) {
        float v[NV][V];
        float total = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            next[i].get(v[i]);
#pragma unroll
            for (int j = 0; j < V; ++j) total += v[i][j];
        }
        fetch(r + step);
        const float mean = sum.template of<WARP>(make_float2(total, 0.f)).x * P.inv_width;
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * span + tid) * V;
                float a = 0.f;
#pragma unroll
                for (int j = 0; j < V; ++j) a = fmaxf(a, finite_abs(v[i][j]));
#pragma unroll
                for (int d = 8; d; d >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
                if (c >= width) continue;
                const unsigned s = scale_byte(a);
                if constexpr (V == 8) *reinterpret_cast<uint2 *>(P.kq + r * P.kqs + c) = pack_eight(v[i], inverse_scale(s));
                if ((tid & 15) == 0) P.kscale[r * P.kss + c / TAD_BLOCK8] = (uint8_t)s;
            }
        }
        float squares = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool live = (i * span + tid) * V < width;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[i][j] -= mean;
                if (live) squares += v[i][j] * v[i][j];
            }
        }
        const float rstd = rsqrtf(sum.template of<WARP>(make_float2(squares, 0.f)).x * P.inv_width + P.eps);
        if (tid == 0) {
            if (P.mean) P.mean[r] = mean;
            if (P.rstd) P.rstd[r] = rstd;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * span + tid) * V;
            if (c >= width) continue;
            float o[V], wr[V], br[V];
            if constexpr (!HOLD) {
                load_vector<V>(wr, P.w, P.w_type, c, width, 1.f);
                load_vector<V>(br, P.b, P.b_type, c, width, 0.f);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = fmaf(v[i][j] * rstd, HOLD ? w[HOLD ? i : 0][j] : wr[j], HOLD ? b[HOLD ? i : 0][j] : br[j]);
            store_typed<V>(P.y, P.y_type, r * P.ys + c, o);
        }
    }
}

// rows of any length: three passes over the row, the second and third from L2
template <class T>
__global__ void __launch_bounds__(LARGE)
tad_norm_forward_long_kernel(const Params P)
{
    __shared__ float2 box[2][32];
    tad_wait_previous();
    Sum sum{box, 0};
    for (int64_t r = blockIdx.x; r < P.n_rows; r += gridDim.x) {
        const T *__restrict__ x = static_cast<const T *>(P.x) + r * P.xs;
        float a = 0.f;
#pragma unroll 8
        for (int c = threadIdx.x; c < P.width; c += LARGE) a += to_float(x[c]);
        const float mean = sum.of<false>(make_float2(a, 0.f)).x * P.inv_width;
        a = 0.f;
#pragma unroll 8
        for (int c = threadIdx.x; c < P.width; c += LARGE) { const float d = to_float(x[c]) - mean; a += d * d; }
        const float rstd = rsqrtf(sum.of<false>(make_float2(a, 0.f)).x * P.inv_width + P.eps);
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
struct Source<Packed8, 8> {
    uint2 q;
    unsigned s;
    __device__ __forceinline__ void zero() { q = make_uint2(0, 0); s = 127; }
    __device__ __forceinline__ void load(const Params &P, int64_t r, int c)
    {
        q = *reinterpret_cast<const uint2 *>(P.q + r * P.qs + c);
        s = P.scale[r * P.ss + c / TAD_BLOCK8];
    }
    __device__ __forceinline__ void get(float (&v)[8]) const { unpack_eight(q, scale_of(s), v); }
};
template <>
struct Source<Packed8, 1> {
    uint8_t q, s;
    __device__ __forceinline__ void zero() { q = 0; s = 127; }
    __device__ __forceinline__ void load(const Params &P, int64_t r, int c) { q = P.q[r * P.qs + c]; s = P.scale[r * P.ss + c / TAD_BLOCK8]; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = from_e4m3x2(q).x * scale_of(s); }
};

template <class S, class T, int V, bool WARP, bool HOLD>
__global__ void __launch_bounds__(HOLD ? SMALL : LARGE, HOLD ? 2 : 1)
tad_norm_backward_kernel(const Params P)
{
    constexpr int NV = E / V;
    __shared__ float2 box[2][32];
    __shared__ float join[WARP ? SMALL / 32 : 1][WARP ? 32 * V : 1];
    tad_wait_previous();
    Sum sum{box, 0};
    const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, span = WARP ? 32 : blockDim.x;
    const int64_t step = WARP ? (int64_t)gridDim.x * (SMALL / 32) : gridDim.x;
    int64_t r = WARP ? (int64_t)blockIdx.x * (SMALL / 32) + (threadIdx.x >> 5) : blockIdx.x;
    const T *__restrict__ dy = static_cast<const T *>(P.dy);
    const int width = P.width;
    float w[HOLD ? NV : 1][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if constexpr (HOLD) load_vector<V>(w[i], P.w, P.w_type, (i * span + tid) * V, width, 1.f);
#pragma unroll
        for (int j = 0; j < V; ++j) dw[i][j] = db[i][j] = 0.f;
    }
    Source<S, V> nx[NV];
    Piece<T, V> ndy[NV];
    float nmean = 0.f, nrstd = 0.f;
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * span + tid) * V;
            nx[i].zero();
            ndy[i].zero();
            if (row < P.n_rows && c < width) {
                nx[i].load(P, row, c);
                ndy[i].load(dy + row * P.dys + c);
            }
        }
        if (row < P.n_rows) { nmean = P.mean[row]; nrstd = P.rstd[row]; }
    };
    fetch(r);
    for (; r < P.n_rows; r += step) {
        float xh[NV][V], d[NV][V];
        const float mean = nmean, rstd = nrstd;
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * span + tid) * V;
            nx[i].get(xh[i]);
            ndy[i].get(d[i]);
            float wr[V];
            if constexpr (!HOLD) load_vector<V>(wr, P.w, P.w_type, c, width, 1.f);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                xh[i][j] = (xh[i][j] - mean) * rstd;
                if (c >= width) xh[i][j] = 0.f;            // (an infinite rstd or a NaN mean must not reach the sums from behind the row)
                dw[i][j] += d[i][j] * xh[i][j];
                db[i][j] += d[i][j];
                d[i][j] *= HOLD ? w[HOLD ? i : 0][j] : wr[j];
                s.x += d[i][j];
                s.y += d[i][j] * xh[i][j];
            }
        }
        fetch(r + step);
        s = sum.template of<WARP>(s);
        const float c1 = s.x * P.inv_width, c2 = s.y * P.inv_width;
        if (P.dx) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * span + tid) * V;
                if (c >= width) continue;
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = rstd * (d[i][j] - c1 - xh[i][j] * c2);
                store_typed<V>(P.dx, P.dx_type, r * P.dxs + c, o);
            }
        }
    }
    if (!P.planes) return;
    float *plane = P.planes + (size_t)blockIdx.x * 2 * width;
    if constexpr (WARP) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < V; ++j) join[threadIdx.x >> 5][tid * V + j] = k ? db[i][j] : dw[i][j];
                __syncthreads();
                for (int e = threadIdx.x; e < 32 * V; e += SMALL) {
                    const int c = i * 32 * V + e;
                    float a = 0.f;
#pragma unroll
                    for (int q = 0; q < SMALL / 32; ++q) a += join[q][e];
                    if (c < width) plane[(size_t)k * width + c] = a;
                }
            }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = (i * span + tid) * V + j;
                if (c < width) { plane[c] = dw[i][j]; plane[(size_t)width + c] = db[i][j]; }
            }
    }
}

// rows of any length: the sums and dx of a row by a block, its columns by tad_norm_columns_kernel
template <class S, class T>
__global__ void __launch_bounds__(LARGE)
tad_norm_backward_long_kernel(const Params P)
{
    __shared__ float2 box[2][32];
    tad_wait_previous();
    Sum sum{box, 0};
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
        s = sum.of<false>(s);
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

struct Shape { int threads; int64_t most; bool warp, hold, is_long; };          // most: blocks that a B200 runs at a time
Shape shape_of(int64_t width, int sm_threads)
{
    Shape s{};
    s.warp = width <= WARP_WIDTH;
    s.is_long = width > HELD;
    s.threads = s.warp ? SMALL : s.is_long ? LARGE : (int)((width + 32 * E - 1) / (32 * E)) * 32;
    s.hold = s.threads <= SMALL;
    s.most = (int64_t)SMS * std::max(1, std::min(32, sm_threads / s.threads));
    return s;
}
constexpr int FORWARD_THREADS = 768, BACKWARD_THREADS = 512;        // of an SM that the registers of the kernels allow

// planes of partial sums of the backward pass: one a block
int64_t planes_of(int64_t n_rows, int64_t width)
{
    const Shape s = shape_of(width, BACKWARD_THREADS);
    if (s.is_long) return std::max<int64_t>(1, std::min<int64_t>(n_rows, 64));
    const int64_t blocks = s.warp ? (n_rows + SMALL / 32 - 1) / (SMALL / 32) : n_rows;
    return std::max<int64_t>(1, std::min(blocks, s.most));
}

template <class T>
cudaError_t forward(const Params &P, const Shape &s, bool eights, bool keep, cudaStream_t stream)
{
    if (s.is_long) return tad_launch(tad_norm_forward_long_kernel<T>, (unsigned)std::min<int64_t>(P.n_rows, 2 * SMS), LARGE, 0, stream, P);
    const int64_t want = s.warp ? (P.n_rows + SMALL / 32 - 1) / (SMALL / 32) : P.n_rows;
    const unsigned blocks = (unsigned)std::min(want, s.most);
    auto kernel = tad_norm_forward_kernel<T, 1, true, true, false>;
    if (eights && keep) kernel = s.warp ? tad_norm_forward_kernel<T, 8, true, true, true> : s.hold ? tad_norm_forward_kernel<T, 8, false, true, true> : tad_norm_forward_kernel<T, 8, false, false, true>;
    else if (eights) kernel = s.warp ? tad_norm_forward_kernel<T, 8, true, true, false> : s.hold ? tad_norm_forward_kernel<T, 8, false, true, false> : tad_norm_forward_kernel<T, 8, false, false, false>;
    else if (!s.warp) kernel = s.hold ? tad_norm_forward_kernel<T, 1, false, true, false> : tad_norm_forward_kernel<T, 1, false, false, false>;
    return tad_launch(kernel, blocks, s.threads, 0, stream, P);
}

template <class S, class T>
cudaError_t backward(const Params &P, const Shape &s, bool eights, int64_t planes, cudaStream_t stream)
{
    if (s.is_long) {
        cudaError_t e = cudaSuccess;
        if (P.dx) e = tad_launch(tad_norm_backward_long_kernel<S, T>, (unsigned)std::min<int64_t>(P.n_rows, 2 * SMS), LARGE, 0, stream, P);
        if (e == cudaSuccess && P.planes)
            e = tad_launch(tad_norm_columns_kernel<S, T>, dim3((unsigned)((P.width + SMALL - 1) / SMALL), (unsigned)planes), SMALL, 0, stream, P, (P.n_rows + planes - 1) / planes);
        return e;
    }
    auto kernel = tad_norm_backward_kernel<S, T, 1, true, true>;
    if (eights) kernel = s.warp ? tad_norm_backward_kernel<S, T, 8, true, true> : s.hold ? tad_norm_backward_kernel<S, T, 8, false, true> : tad_norm_backward_kernel<S, T, 8, false, false>;
    else if (!s.warp) kernel = s.hold ? tad_norm_backward_kernel<S, T, 1, false, true> : tad_norm_backward_kernel<S, T, 1, false, false>;
    return tad_launch(kernel, (unsigned)planes, s.threads, 0, stream, P);
}

}  // namespace

extern "C" {

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
    if (!(eps >= 0.f)) return bad("layernorm_forward: eps is negative or NaN");
    if (n_rows == 0) return TAD_OK;
    if (width == 0) {
        if (mean || rstd) return bad("layernorm_forward: rows of no elements have no mean");
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
    const Shape s = shape_of(width, FORWARD_THREADS);
    const bool eights = width % 8 == 0 && by_eights(x) && by_eights(y), keep = checkpoint && eights && !s.is_long;
    if (keep) { P.kq = checkpoint->q; P.kqs = checkpoint->q_stride; P.kscale = checkpoint->scale; P.kss = checkpoint->scale_stride; }
    else if (checkpoint && (st = tad_launch_pack8(x, n_rows, width, checkpoint, stream))) return st;
    cudaError_t e = cudaSuccess;
    TAD_WITH_TYPE(x->type, T, e = forward<T>(P, s, eights, keep, stream));
    return launched("layer norm", e);
}

size_t tad_layernorm_workspace_bytes(int64_t n_rows, int64_t width)
{
    if (n_rows <= 0 || width <= 0 || n_rows >= MAX_ROWS || width >= MAX_WIDTH) return 0;
    return ((size_t)planes_of(n_rows, width) * 2 * (size_t)width * 4 + 255) & ~size_t(255);
}

tad_status tad_layernorm_backward(const tad_rows *dy, const tad_rows *x, const tad_packed *checkpoint, int64_t n_rows, int64_t width,
                                  const tad_rows *weight, const float *mean, const float *rstd, const tad_rows *dx,
                                  const tad_rows *dweight, const tad_rows *dbias, void *workspace, size_t workspace_bytes,
                                  void *cuda_stream)
{
    tad_status st;
    if ((st = check_sizes("layernorm_backward", n_rows, width)) || (st = check_rows("layernorm_backward: dy", dy, n_rows, width))) return st;
    if (!x == !checkpoint) return bad("layernorm_backward: x or a checkpoint of it, one of the two");
    if (x && (st = check_rows("layernorm_backward: x", x, n_rows, width))) return st;
    if (checkpoint && (st = check_packed("layernorm_backward: checkpoint", checkpoint, n_rows, width))) return st;
    if (weight && (st = check_rows("layernorm_backward: weight", weight, 1, width, true))) return st;
    if (dx && (st = check_rows("layernorm_backward: dx", dx, n_rows, width))) return st;
    if (dweight && (st = check_rows("layernorm_backward: dweight", dweight, 1, width, true))) return st;
    if (dbias && (st = check_rows("layernorm_backward: dbias", dbias, 1, width, true))) return st;
    if (width == 0) return TAD_OK;
    if (n_rows > 0 && (!mean || !rstd)) return bad("layernorm_backward: NULL mean or rstd");
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
        const Shape s = shape_of(width, BACKWARD_THREADS);
        const bool eights = width % 8 == 0 && by_eights(dy) && (!x || by_eights(x)) && (!dx || by_eights(dx));
        planes = planes_of(n_rows, width);
        TAD_WITH_TYPE(dy->type, T, {
            if (!x) e = backward<Packed8, T>(P, s, eights, planes, stream);
            else TAD_WITH_TYPE(x->type, S, e = backward<S, T>(P, s, eights, planes, stream));
        });
    }
    if (e == cudaSuccess && sums)
        e = tad_launch(tad_norm_planes_kernel, (unsigned)((2 * width + 31) / 32), 1024, 0, stream, static_cast<const float *>(workspace), (int)planes, (int)width,
                       dweight ? dweight->data : nullptr, dweight ? dweight->type : 0, dbias ? dbias->data : nullptr, dbias ? dbias->type : 0);
    return launched("layer norm backward", e);
}

}  // extern "C"
