// Helpers shared by the row operators (norm, 8-bit rows, loss, clipping):
// groups of elements loaded as floats and stored rounded once, sums over the
// warps that share a row, argument checks.
#pragma once

#include "ember_device.cuh"
#include "ember_internal.h"

namespace ember {
namespace rows {

constexpr int kMaxRowCols = 32768;  // widest row of the norm operators

struct bf16_t { unsigned short u; };

// A group of VEC elements as it is in memory: 8 (16 bytes of bf16, 32 of fp32,
// one access each) or 1.  Kept packed between the load and its uses.  The
// loads are volatile so that a thread's loads are issued together, before the
// first use; no kernel stores where another thread's later load may read.
template <typename T, int VEC> struct Raw;
template <> struct Raw<bf16_t, 8> { uint4 v; };
template <> struct Raw<bf16_t, 1> { unsigned short v; };
template <> struct Raw<float, 8> { float4 a, b; };
template <> struct Raw<float, 1> { float v; };

template <typename T, int VEC>
__device__ __forceinline__ Raw<T, VEC> load_raw(const T *p)
{
    Raw<T, VEC> r;
    if constexpr (sizeof(T) == 2 && VEC == 8)
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r.v.x), "=r"(r.v.y), "=r"(r.v.z), "=r"(r.v.w)
                     : "l"(p));
    else if constexpr (sizeof(T) == 2)
        r.v = p->u;
    else if constexpr (VEC == 8) {
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(r.a.x), "=f"(r.a.y), "=f"(r.a.z), "=f"(r.a.w), "=f"(r.b.x), "=f"(r.b.y), "=f"(r.b.z),
                       "=f"(r.b.w)
                     : "l"(p));
    } else
        r.v = *p;
    return r;
}

template <typename T, int VEC>
__device__ __forceinline__ Raw<T, VEC> zero_raw()
{
    Raw<T, VEC> r;
    if constexpr (sizeof(T) == 2 && VEC == 8)
        r.v = make_uint4(0, 0, 0, 0);
    else if constexpr (VEC == 8) {
        r.a = make_float4(0.f, 0.f, 0.f, 0.f);
        r.b = r.a;
    } else
        r.v = 0;
    return r;
}

template <typename T, int VEC>
__device__ __forceinline__ void unpack(const Raw<T, VEC> &r, float (&f)[VEC])
{
    if constexpr (sizeof(T) == 2 && VEC == 8) {
        const unsigned u[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = dev::bf16_lo(u[k]);
            f[2 * k + 1] = dev::bf16_hi(u[k]);
        }
    } else if constexpr (sizeof(T) == 2)
        f[0] = __uint_as_float((unsigned)r.v << 16);
    else if constexpr (VEC == 8) {
        f[0] = r.a.x; f[1] = r.a.y; f[2] = r.a.z; f[3] = r.a.w;
        f[4] = r.b.x; f[5] = r.b.y; f[6] = r.b.z; f[7] = r.b.w;
    } else
        f[0] = r.v;
}

// Two floats rounded to nearest even and packed, the first in the low half.
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned *>(&v);
}

template <typename T, int VEC>
__device__ __forceinline__ void store_group(T *p, const float (&f)[VEC])
{
    if constexpr (sizeof(T) == 2 && VEC == 8)
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]),
                                                   pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    else if constexpr (sizeof(T) == 2)
        p->u = dev::f2bf(f[0]);
    else if constexpr (VEC == 8)
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]),
                     "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7])
                     : "memory");
    else
        *p = f[0];
}

// Gains (fp32, bf16 or none) of a group of columns.
template <int VEC>
__device__ __forceinline__ void load_gain(const void *gain, int gbf16, int64_t col, float (&g)[VEC])
{
    if (gain == nullptr) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            g[e] = 1.f;
    } else if (gbf16)
        unpack<bf16_t, VEC>(load_raw<bf16_t, VEC>(static_cast<const bf16_t *>(gain) + col), g);
    else
        unpack<float, VEC>(load_raw<float, VEC>(static_cast<const float *>(gain) + col), g);
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1)
        v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// NaN is larger than everything else here, so that it survives a maximum.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max_nan(float v)
{
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1)
        v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Pairs of floats in one instruction.
struct f2 {
    unsigned long long v;
};
__device__ __forceinline__ f2 make2(float x, float y)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void split2(f2 a, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(a.v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ float sum2(f2 a)
{
    float x, y;
    split2(a, x, y);
    return x + y;
}
// A group of 8 as pairs.
template <typename T>
__device__ __forceinline__ void unpack2(const Raw<T, 8> &r, f2 (&f)[4])
{
    float e[8];
    unpack<T, 8>(r, e);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        f[k] = make2(e[2 * k], e[2 * k + 1]);
}
template <typename T>
__device__ __forceinline__ void store_group2(T *p, const f2 (&f)[4])
{
    float e[8];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        split2(f[k], e[2 * k], e[2 * k + 1]);
    store_group<T, 8>(p, e);
}

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool dtype_ok(int t) { return t == EMBER_F32 || t == EMBER_BF16; }
inline size_t elem_size(int t) { return t == EMBER_BF16 ? 2 : 4; }
// Whether every row of a matrix of this type starts on a group of 8 elements.
inline bool grouped(const void *p, int64_t ld, int dtype)
{
    return p == nullptr || (aligned(p, 8 * elem_size(dtype)) && ld % 8 == 0);
}
inline ember_status launched(cudaError_t e)
{
    if (e == cudaSuccess)
        return EMBER_OK;
    cudaGetLastError();  // the error is returned, not left for the next call to find
    return EMBER_ERR_CUDA;
}

}  // namespace rows
}  // namespace ember
