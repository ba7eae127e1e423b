// Rows of 32- and 16-bit elements and of packed 8-bit blocks: descriptors as the kernels take them, their checks on the host,
// loads and stores of eight elements or of one, packing and unpacking.  Shared by norm.cu, embed.cu, pack8.cu and product8.cu.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cstdio>
#include <type_traits>

#include "../../include/tad.h"
#include "launch.h"

namespace tad { void set_error(const char *m) noexcept; }

// waits in the kernels launched from now on count as run out (tad_debug_lost_waits; norm.cu)
namespace tadr { extern std::atomic<int> lost_waits; }

namespace tadr {

constexpr int64_t MAX_WIDTH = int64_t(1) << 24, MAX_ROWS = int64_t(1) << 31;
constexpr int SMS = 148;                                  // of a B200: what grids are made for (any number is right)

// ---- host: checks ----

// (nothing here allocates: an exception may not leave the C entry points)
inline tad_status refuse(tad_status status, const char *what, const char *why) noexcept
{
    char text[256];
    std::snprintf(text, sizeof text, "%s: %s", what, why);
    tad::set_error(text);
    return status;
}
inline tad_status bad(const char *what, const char *why) noexcept { return refuse(TAD_ERR_INVALID_ARG, what, why); }

inline tad_status check_sizes(const char *what, int64_t n_rows, int64_t width)
{
    if (n_rows < 0 || width < 0) return bad(what, "negative size");
    if (n_rows >= MAX_ROWS || width >= MAX_WIDTH) return refuse(TAD_ERR_UNSUPPORTED, what, "2^31 rows or a width of 2^24 and more");
    return TAD_OK;
}

inline size_t type_size(int type) { return type == TAD_F32 ? 4 : 2; }

// vector: one row, the stride is not looked at
inline tad_status check_rows(const char *what, const tad_rows *m, int64_t n_rows, int64_t width, bool vector = false)
{
    if (!m) return bad(what, "NULL matrix");
    if (m->type != TAD_F32 && m->type != TAD_BF16 && m->type != TAD_F16) return bad(what, "unknown element type");
    if (m->reserved != 0) return bad(what, "reserved field is not zero");
    if (!vector && m->stride < width) return bad(what, "stride below the width");
    if (n_rows == 0 || width == 0) return TAD_OK;
    if (!m->data) return bad(what, "NULL data");
    if (reinterpret_cast<uintptr_t>(m->data) % type_size(m->type)) return bad(what, "data not aligned to its element");
    return TAD_OK;
}

inline int64_t blocks_of(int64_t width) { return (width + TAD_BLOCK8 - 1) / TAD_BLOCK8; }

inline tad_status check_packed(const char *what, const tad_packed *m, int64_t n_rows, int64_t width)
{
    if (!m) return bad(what, "NULL packed matrix");
    if (m->q_stride < width || m->scale_stride < blocks_of(width)) return bad(what, "stride below the width");
    if (m->q_stride % 16 || m->scale_stride % 4) return bad(what, "q_stride must be a multiple of 16, scale_stride of 4");
    if (n_rows == 0 || width == 0) return TAD_OK;
    if (!m->q || !m->scale) return bad(what, "NULL data");
    if (reinterpret_cast<uintptr_t>(m->q) % 16 || reinterpret_cast<uintptr_t>(m->scale) % 4) return bad(what, "q must be 16-byte aligned, scale 4-byte");
    return TAD_OK;
}

inline tad_status check_room(const char *what, const void *workspace, size_t bytes, size_t need)
{
    if (need && (!workspace || bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)))
        return refuse(TAD_ERR_WORKSPACE, what, "workspace missing, too small or not 256-byte aligned");
    return TAD_OK;
}

inline tad_status launched(const char *what, cudaError_t e)
{
    if (e == cudaSuccess) return TAD_OK;
    char launch[64];
    std::snprintf(launch, sizeof launch, "%s launch failed", what);
    return refuse(TAD_ERR_CUDA, launch, cudaGetErrorString(e));
}

// rows that eight elements at a time can be read from and written to by one access of 16 or, fp32, 32 bytes
inline bool by_eights(const tad_rows *m) { return reinterpret_cast<uintptr_t>(m->data) % (8 * type_size(m->type)) == 0 && m->stride % 8 == 0; }

// ---- device: elements ----

template <class T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float(float v) { return v; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }

// V = 8 or 1 elements as they lie in memory
template <class T, int V> struct Piece;
template <class T> struct Piece<T, 1> {
    T e;
    __device__ __forceinline__ void load(const T *p) { e = *p; }
    __device__ __forceinline__ void zero() { e = from_float<T>(0.f); }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_float(e); }
    __device__ __forceinline__ void set(const float (&v)[1]) { e = from_float<T>(v[0]); }
    __device__ __forceinline__ void store(T *p) const { *p = e; }
};
template <> struct Piece<float, 8> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) { a = reinterpret_cast<const float4 *>(p)[0]; b = reinterpret_cast<const float4 *>(p)[1]; }
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float (&v)[8]) const { v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w; }
    __device__ __forceinline__ void set(const float (&v)[8]) { a = make_float4(v[0], v[1], v[2], v[3]); b = make_float4(v[4], v[5], v[6], v[7]); }
    // (one store of 32 bytes: two of 16 leave half of every sector to the second; 8192 x 8192 unpacked to fp32 70 us for 52)
    __device__ __forceinline__ void store(float *p) const
    {
        asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(a.x), "f"(a.y), "f"(a.z), "f"(a.w), "f"(b.x), "f"(b.y), "f"(b.z), "f"(b.w) : "memory");
    }
};
template <> struct Piece<__nv_bfloat16, 8> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { a = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(w[j] << 16); v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        unsigned w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
            w[j] = *reinterpret_cast<const unsigned *>(&h);
        }
        a = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = a; }
};
template <> struct Piece<__half, 8> {
    uint4 a;
    __device__ __forceinline__ void load(const __half *p) { a = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[j]));
            v[2 * j] = f.x; v[2 * j + 1] = f.y;
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        unsigned w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __half2 h = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
            w[j] = *reinterpret_cast<const unsigned *>(&h);
        }
        a = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void store(__half *p) const { *reinterpret_cast<uint4 *>(p) = a; }
};

// an element of a vector whose type is known at run time only (weights: read once a block)
__device__ __forceinline__ float element(const void *p, int type, int64_t i)
{
    if (type == TAD_F32) return static_cast<const float *>(p)[i];
    if (type == TAD_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(static_cast<const __half *>(p)[i]);
}
__device__ __forceinline__ void put_element(void *p, int type, int64_t i, float v)
{
    if (type == TAD_F32) static_cast<float *>(p)[i] = v;
    else if (type == TAD_BF16) static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half *>(p)[i] = __float2half_rn(v);
}

// ---- device: 8-bit blocks ----

// |x| as it counts for the scale of a block: infinities and NaNs do not
__device__ __forceinline__ float finite_abs(float x) { const float a = fabsf(x); return a <= 3.402823466e38f ? a : 0.f; }

// exponent byte of a block's scale: k the least integer >= -126 with a <= 448 2^k = 1.75 2^(k + 8), 0 for a = 0
__device__ __forceinline__ unsigned scale_byte(float a)
{
    const unsigned u = __float_as_uint(a), e = u >> 23;                      // (a >= 0: no sign)
    const int k = (int)e - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return a > 0.f ? (unsigned)(max(k, -126) + 127) : 127u;
}
// 2^(127 - b) for a byte b of scale_byte(): 1 <= b <= 247, so the quotient x / 2^k is this exact product
__device__ __forceinline__ float inverse_scale(unsigned b) { return __uint_as_float((254u - b) << 23); }
// 2^(b - 127): 0 is 2^-127, a subnormal number; 255 stands for NaN, here it is an infinity
__device__ __forceinline__ float scale_or_infinity(unsigned b) { return __uint_as_float(max(b << 23, 0x00400000u)); }
__device__ __forceinline__ float scale_of(unsigned b) { return b == 255u ? __uint_as_float(0x7fffffffu) : scale_or_infinity(b); }

// two values, already divided by their scale, to e4m3 (the first in the low byte); an infinity would become 448
__device__ __forceinline__ unsigned to_e4m3x2(float lo, float hi) { return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ float2 from_e4m3x2(unsigned two)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
// infinities as NaNs: e4m3 has none, and the conversion would make them 448
__device__ __forceinline__ float no_infinity(float x) { return isinf(x) ? __uint_as_float(0x7fffffffu) : x; }

__device__ __forceinline__ void unpack_eight(uint2 q, float s, float (&v)[8])
{
    const unsigned h[4] = {q.x & 0xffffu, q.x >> 16, q.y & 0xffffu, q.y >> 16};
#pragma unroll
    for (int j = 0; j < 4; ++j) { const float2 f = from_e4m3x2(h[j]); v[2 * j] = f.x * s; v[2 * j + 1] = f.y * s; }
}

// Sixteen elements as they lie in memory, zeros behind the row.  The magnitudes of 16-bit types are compared as integers, two at a time;
// infinities and NaNs are above all finite numbers there.
template <class T>
struct Sixteen {
    unsigned w[8];
    static constexpr unsigned INF = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
    __device__ __forceinline__ void load(const T *__restrict__ row, int c, int width)
    {
        if (c + 16 <= width) {
            const uint4 a = reinterpret_cast<const uint4 *>(row + c)[0], b = reinterpret_cast<const uint4 *>(row + c)[1];
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
        } else {
            const unsigned short *h = reinterpret_cast<const unsigned short *>(row);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                w[j] = (c + 2 * j < width ? h[c + 2 * j] : 0u) | (c + 2 * j + 1 < width ? (unsigned)h[c + 2 * j + 1] << 16 : 0u);
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 0;
    }
    __device__ __forceinline__ float2 pair(int j) const
    {
        if (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2 *>(&w[j]));
        return make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    }
    // the largest magnitude of the block's eight lanes
    __device__ __forceinline__ float most(bool &odd) const
    {
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = __vmaxu2(m, w[j] & 0x7fff7fffu);
#pragma unroll
        for (int d = 4; d; d >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, d));
        m = max(m & 0xffffu, m >> 16);
        odd = m >= INF;
        if (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)m));
        return __uint_as_float(m << 16);
    }
    // The block's eight lanes pack it together; byte: its scale.  Infinities and NaNs are looked for once a block and a warp.
    __device__ __forceinline__ uint4 pack(unsigned &byte) const
    {
        bool odd;
        float a = most(odd);
        const bool rare = __any_sync(0xffffffffu, odd);
        if (rare) {
            a = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) { const float2 f = pair(j); a = fmaxf(a, fmaxf(finite_abs(f.x), finite_abs(f.y))); }
#pragma unroll
            for (int d = 4; d; d >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
        }
        byte = scale_byte(a);
        const float inv = inverse_scale(byte);
        unsigned u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float2 f = pair(2 * j), g = pair(2 * j + 1);
            if (rare) { f.x = no_infinity(f.x); f.y = no_infinity(f.y); g.x = no_infinity(g.x); g.y = no_infinity(g.y); }
            u[j] = to_e4m3x2(f.x * inv, f.y * inv) | (to_e4m3x2(g.x * inv, g.y * inv) << 16);
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
};
template <>
struct Sixteen<float> {
    float v[16];
    __device__ __forceinline__ void load(const float *__restrict__ row, int c, int width)
    {
        if (c + 16 <= width) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 a = reinterpret_cast<const float4 *>(row + c)[j];
                v[4 * j] = a.x; v[4 * j + 1] = a.y; v[4 * j + 2] = a.z; v[4 * j + 3] = a.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = c + j < width ? row[c + j] : 0.f;
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = 0.f;
    }
    __device__ __forceinline__ float2 pair(int j) const { return make_float2(v[2 * j], v[2 * j + 1]); }
    __device__ __forceinline__ float most(bool &odd) const
    {
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
#pragma unroll
        for (int d = 4; d; d >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
        odd = m >= 0x7f800000u;
        return __uint_as_float(m);
    }
    // The block's eight lanes pack it together; byte: its scale.  Infinities and NaNs are looked for once a block and a warp.
    __device__ __forceinline__ uint4 pack(unsigned &byte) const
    {
        bool odd;
        float a = most(odd);
        const bool rare = __any_sync(0xffffffffu, odd);
        if (rare) {
            a = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) { const float2 f = pair(j); a = fmaxf(a, fmaxf(finite_abs(f.x), finite_abs(f.y))); }
#pragma unroll
            for (int d = 4; d; d >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, d));
        }
        byte = scale_byte(a);
        const float inv = inverse_scale(byte);
        unsigned u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float2 f = pair(2 * j), g = pair(2 * j + 1);
            if (rare) { f.x = no_infinity(f.x); f.y = no_infinity(f.y); g.x = no_infinity(g.x); g.y = no_infinity(g.y); }
            u[j] = to_e4m3x2(f.x * inv, f.y * inv) | (to_e4m3x2(g.x * inv, g.y * inv) << 16);
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
};

}  // namespace tadr

// CALL(T) with the element type of a tad_type
#define TAD_WITH_TYPE(type, T, ...)                                                        \
    do {                                                                                   \
        if ((type) == TAD_F32) { using T = float; __VA_ARGS__; }                           \
        else if ((type) == TAD_BF16) { using T = __nv_bfloat16; __VA_ARGS__; }             \
        else { using T = __half; __VA_ARGS__; }                                            \
    } while (0)
