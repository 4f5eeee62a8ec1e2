// Residual addition with the root-mean-square norm, its output in the
// input's type or in 8 bits with a scale per row, its gradients, and the
// same 8-bit rows of any matrix.
//
//   s = x + residual                     (h = s rounded to the residual's type)
//   y_j = gain_j s_j / sqrt(mean_j s_j^2 + eps)
//   scale = max_j |y_j| / 127,  q_j = y_j / scale rounded to nearest even
//
// and for the gradients, with n = sqrt(mean_j h_j^2 + eps):
//   dx_j = gain_j dy_j / n - h_j (sum_k gain_k dy_k h_k) / (D n^3) + dres_j
//   dgain_j = sum_t dy_tj h_tj / n_t
//
// Every kernel is bound by HBM: a row is loaded once, stays in registers
// between the sums and the outputs, and each output is written once.  A row
// belongs to `tpr` threads (32 to 1024) of NV groups of VEC elements each, so
// that one barrier joins the warps' sums.  The norm is formed from the sum in
// 32 bits, not from the h that is stored: rounding it first would add the
// error of one bf16 rounding to y.
//
// Measured, of the copy bandwidth (6780 GB/s): norm 8192 x 4096 bf16 with an
// fp32 residual 60.7 us, 0.98; 8192 x 8192 bf16 with residual 79 us, 1.00;
// in 8 bits 79 us, 0.88; backward with dres 89 us, 0.89 (fp32 156 us, 1.02).
// Rows off the 16-byte boundaries: 0.2 to 0.85 (k_rmsnorm_shifted).
#include <type_traits>

#include "ember_rows.cuh"

namespace ember {
namespace {

using namespace rows;

constexpr int kMinBlock = 128;  // threads of a CTA: several short rows share one

// Sums (or NaN-keeping maxima) over the threads of one row.  `part` holds a
// value per warp of the CTA; the warps of a row are added in order, so the
// result does not depend on how many rows share the CTA.
template <bool MAX>
__device__ __forceinline__ float row_reduce(float v, float *part, int tpr)
{
    v = MAX ? warp_max_nan(v) : warp_sum(v);
    if (tpr == 32)
        return v;
    const int w = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0)
        part[w] = v;
    __syncthreads();
    const int nw = tpr >> 5;
    const int w0 = w / nw * nw;
    float r = part[w0];
    for (int k = 1; k < nw; ++k)
        r = MAX ? max_nan(r, part[w0 + k]) : r + part[w0 + k];
    return r;
}

// q = y / scale rounded to fp32 and then to nearest even, |q| <= 127.  A row of
// zeros has the scale 0 and zeros; a row with an infinity or a NaN has the
// scale NaN and zeros, so that what is formed from it is NaN throughout.
struct RowScale {
    float scale, inv;
    bool divide;
};
__device__ __forceinline__ RowScale row_scale(float top)
{
    RowScale s;
    s.divide = false;
    s.scale = top / 127.f;
    s.inv = 0.f;
    if (!(top <= 3.402823466e38f)) {  // infinity or NaN
        s.scale = __uint_as_float(0x7FC00000u);
    } else if (s.scale >= 1e-25f) {
        s.inv = 1.f / s.scale;
    } else if (s.scale > 0.f) {  // 1 / scale may overflow, scale itself or a remainder be subnormal
        s.divide = true;
    }
    return s;
}
// The codes of VEC values, in the low bytes: adding 1.5 2^23 leaves a value
// rounded to an integer, nearest even, in the low bits of the fp32 number.  The
// quotient is y inv with one correction by its remainder (Markstein's division):
// what is rounded once more is the quotient to within 2^-22 of its last place, so
// a value next to a tie falls to its side.  (By y inv alone, which is off by up to
// 2^-17, one code in 10^5 differs.)  |quotient| is at most 127 (1 + 2^-23), so
// no bound is needed there.
template <int VEC>
__device__ __forceinline__ void quants(const float (&y)[VEC], const RowScale &s, unsigned (&q)[VEC])
{
    if (s.divide) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            q[e] = __float_as_uint(fminf(fmaxf(y[e] / s.scale, -127.f), 127.f) + 12582912.f);
        return;
    }
    if (s.inv == 0.f) {  // zeros, also where y is infinite or NaN
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            q[e] = 0;
        return;
    }
    // pairs: without a test per value 8192 x 8192 bf16 take 48 us, with one 61
    const f2 inv = make2(s.inv, s.inv), minus = make2(-s.scale, -s.scale), magic = make2(12582912.f, 12582912.f);
#pragma unroll
    for (int e = 0; e < VEC; e += 2) {
        const f2 v = make2(y[e], VEC > 1 ? y[e + (VEC > 1)] : 0.f);
        const f2 guess = mul2(v, inv);
        float lo, hi;
        split2(add2(fma2(fma2(guess, minus, v), inv, guess), magic), lo, hi);
        q[e] = __float_as_uint(lo);
        if constexpr (VEC > 1)
            q[e + 1] = __float_as_uint(hi);
    }
}

template <int VEC>
__device__ __forceinline__ void store_q(int8_t *p, const float (&y)[VEC], const RowScale &s)
{
    unsigned q[VEC];
    quants<VEC>(y, s, q);
    if constexpr (VEC == 8) {
        unsigned u[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            u[k] = __byte_perm(__byte_perm(q[4 * k], q[4 * k + 1], 0x0040),
                               __byte_perm(q[4 * k + 2], q[4 * k + 3], 0x0040), 0x5410);
        *reinterpret_cast<uint2 *>(p) = make_uint2(u[0], u[1]);
    } else
        *p = (int8_t)(q[0] & 0xff);
}

struct NormArgs {
    const void *x, *res, *gain;
    void *h, *y;  // y: the output in x's type, or int8
    float *scales;
    int64_t ldx, ldr, ldh, ldy, T;
    int D, tpr, gbf16;
    float eps;
};

enum { kOutSame = 0, kOutInt = 1 };

// NORM = false: the rows themselves in 8 bits, without a norm.
template <typename XT, typename RT, bool RES, bool NORM, int OUT, int VEC, int NV, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) k_rmsnorm(NormArgs a)
{
    __shared__ float part[2][32];
    const int rpc = blockDim.x / a.tpr;
    const int64_t row = (int64_t)blockIdx.x * rpc + threadIdx.x / a.tpr;
    const int lane = threadIdx.x % a.tpr;
    const bool live = row < a.T;
    dev::grid_dep_wait();
    dev::grid_dep_launch();

    float s[NV][VEC];
    float ss = 0.f;
    const XT *x = static_cast<const XT *>(a.x) + row * a.ldx;
    Raw<XT, VEC> rx[NV];
    Raw<RT, VEC> rr[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int col = (k * a.tpr + lane) * VEC;
        const bool on = live && col < a.D;
        rx[k] = on ? load_raw<XT, VEC>(x + col) : zero_raw<XT, VEC>();
        if constexpr (RES)
            rr[k] = on ? load_raw<RT, VEC>(static_cast<const RT *>(a.res) + row * a.ldr + col)
                       : zero_raw<RT, VEC>();
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        unpack<XT, VEC>(rx[k], s[k]);
        if constexpr (RES) {
            float r[VEC];
            unpack<RT, VEC>(rr[k], r);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s[k][e] += r[e];
        }
        if constexpr (NORM) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                ss = fmaf(s[k][e], s[k][e], ss);
        }
    }
    if constexpr (RES) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int col = (k * a.tpr + lane) * VEC;
            if (live && col < a.D)
                store_group<RT, VEC>(static_cast<RT *>(a.h) + row * a.ldh + col, s[k]);
        }
    }
    if constexpr (NORM) {
        const float rstd = 1.f / sqrtf(row_reduce<false>(ss, part[0], a.tpr) / (float)a.D + a.eps);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int col = (k * a.tpr + lane) * VEC;
            if (col < a.D) {
                float g[VEC];
                load_gain<VEC>(a.gain, a.gbf16, col, g);
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    s[k][e] = s[k][e] * rstd * g[e];
            }
        }
    }
    if constexpr (OUT == kOutInt) {
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                top = max_nan(top, fabsf(s[k][e]));
        const RowScale sc = row_scale(row_reduce<true>(top, part[1], a.tpr));
        if (!live)
            return;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int col = (k * a.tpr + lane) * VEC;
            if (col < a.D)
                store_q<VEC>(static_cast<int8_t *>(a.y) + row * a.ldy + col, s[k], sc);
        }
        if (lane == 0)
            a.scales[row] = sc.scale;
    } else {
        if (!live)
            return;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int col = (k * a.tpr + lane) * VEC;
            if (col < a.D)
                store_group<XT, VEC>(static_cast<XT *>(a.y) + row * a.ldy + col, s[k]);
        }
    }
}

int round32(int n) { return (n + 31) / 32 * 32; }

// Threads per row: a whole number of warps, at most 1024; each takes nv
// groups.  A power of two when it is below a CTA, so that rows share CTAs.
int threads_per_row(int64_t D, int vec, int nv)
{
    const int need = round32((int)((D + (int64_t)vec * nv - 1) / ((int64_t)vec * nv)));
    if (need >= kMinBlock)
        return need;
    int t = 32;
    while (t < need)
        t *= 2;
    return t;
}

template <typename XT, typename RT, bool RES, bool NORM, int OUT, int VEC, int NV, int MAXT = 1024, int MINB = 1>
cudaError_t go_norm(NormArgs a, cudaStream_t stream)
{
    a.tpr = threads_per_row(a.D, VEC, NV);
    const int block = a.tpr < kMinBlock ? kMinBlock : a.tpr;
    const int64_t rpc = block / a.tpr;
    return launch_k(k_rmsnorm<XT, RT, RES, NORM, OUT, VEC, NV, MAXT, MINB>, dim3((unsigned)((a.T + rpc - 1) / rpc)),
                    dim3(block), 0, stream, true, a);
}

// Long rows of whole groups, one row per CTA at a time.  The rows come through
// a ring of two in shared memory, filled by asynchronous copies; a thread
// copies what it will read itself, so the ring needs no barrier, and the next
// two rows are on their way while one is reduced and written.  A thread has the
// same columns in every row and keeps their gains in registers.
constexpr int kRing = 2;       // rows
constexpr int kRingGroups = 4;  // groups of 8 per thread

__device__ __forceinline__ void copy16(void *smem, const void *p)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(p)
                 : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// This thread's groups of one row of one input into the ring, and one of them back.
template <typename T>
__device__ __forceinline__ void ring_fetch(unsigned char *to, const T *row, int groups)
{
    constexpr int GB = 8 * sizeof(T);
#pragma unroll
    for (int k = 0; k < kRingGroups; ++k) {
        const int g = k * blockDim.x + threadIdx.x;
        if (g < groups) {
#pragma unroll
            for (int b = 0; b < GB; b += 16)
                copy16(to + g * GB + b, reinterpret_cast<const unsigned char *>(row) + g * GB + b);
        }
    }
}
template <typename T>
__device__ __forceinline__ void ring_read(const unsigned char *from, int g, f2 (&f)[4])
{
    const unsigned char *p = from + g * (8 * sizeof(T));
    Raw<T, 8> r;
    if constexpr (sizeof(T) == 2)
        r.v = *reinterpret_cast<const uint4 *>(p);
    else {
        r.a = reinterpret_cast<const float4 *>(p)[0];
        r.b = reinterpret_cast<const float4 *>(p)[1];
    }
    unpack2<T>(r, f);
}

__device__ __forceinline__ void gains2(const void *gain, int gbf16, int groups, f2 (&ga)[kRingGroups][4])
{
#pragma unroll
    for (int k = 0; k < kRingGroups; ++k) {
        const int g = k * blockDim.x + threadIdx.x;
        float e[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (g < groups)
            load_gain<8>(gain, gbf16, g * 8, e);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            ga[k][q] = make2(e[2 * q], e[2 * q + 1]);
    }
}

// A value per warp joined over the CTA; `part` is not written again before
// another barrier.
template <bool MAX>
__device__ __forceinline__ float cta_join(float v, float *part)
{
    v = MAX ? warp_max_nan(v) : warp_sum(v);
    const int nw = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (nw == 1)
        return v;
    if (lane == 0)
        part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < nw ? part[lane] : 0.f;
    return MAX ? warp_max_nan(v) : warp_sum(v);
}

template <typename XT, typename RT, bool RES, int OUT, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) k_rmsnorm_ring(NormArgs a)
{
    extern __shared__ __align__(128) unsigned char ring[];  // [stage][x, residual]
    __shared__ float part[2][2][32];                        // by parity of the row
    const int tid = threadIdx.x, nt = blockDim.x;
    const int groups = a.D / 8;
    const int x_bytes = a.D * (int)sizeof(XT), row_bytes = x_bytes + (RES ? a.D * (int)sizeof(RT) : 0);
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    auto fetch = [&](int64_t row, int stage) {
        if (row < a.T) {
            unsigned char *to = ring + (size_t)stage * row_bytes;
            ring_fetch<XT>(to, static_cast<const XT *>(a.x) + row * a.ldx, groups);
            if constexpr (RES)
                ring_fetch<RT>(to + x_bytes, static_cast<const RT *>(a.res) + row * a.ldr, groups);
        }
        copies_commit();
    };
#pragma unroll
    for (int s = 0; s < kRing; ++s)
        fetch(blockIdx.x + (int64_t)s * gridDim.x, s);
    f2 ga[kRingGroups][4];
    gains2(a.gain, a.gbf16, groups, ga);
    int stage = 0, par = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, par ^= 1) {
        copies_wait<kRing - 1>();
        const unsigned char *from = ring + (size_t)stage * row_bytes;
        f2 s[kRingGroups][4];
        f2 ss = make2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kRingGroups; ++k) {
            const int g = k * nt + tid;
            if (g < groups) {
                ring_read<XT>(from, g, s[k]);
                if constexpr (RES) {
                    f2 r[4];
                    ring_read<RT>(from + x_bytes, g, r);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        s[k][q] = add2(s[k][q], r[q]);
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    s[k][q] = make2(0.f, 0.f);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                ss = fma2(s[k][q], s[k][q], ss);
            if constexpr (RES) {
                if (g < groups)
                    store_group2<RT>(static_cast<RT *>(a.h) + row * a.ldh + g * 8, s[k]);
            }
        }
        fetch(row + (int64_t)kRing * gridDim.x, stage);
        stage = stage + 1 == kRing ? 0 : stage + 1;
        const float rstd = 1.f / sqrtf(cta_join<false>(sum2(ss), part[par][0]) / (float)a.D + a.eps);
        const f2 r2 = make2(rstd, rstd);
#pragma unroll
        for (int k = 0; k < kRingGroups; ++k)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                s[k][q] = mul2(mul2(s[k][q], r2), ga[k][q]);
        if constexpr (OUT == kOutInt) {
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < kRingGroups; ++k)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float x, y;
                    split2(s[k][q], x, y);
                    top = max_nan(top, max_nan(fabsf(x), fabsf(y)));
                }
            const RowScale sc = row_scale(cta_join<true>(top, part[par][1]));
#pragma unroll
            for (int k = 0; k < kRingGroups; ++k) {
                const int g = k * nt + tid;
                if (g < groups) {
                    float y[8];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        split2(s[k][q], y[2 * q], y[2 * q + 1]);
                    store_q<8>(static_cast<int8_t *>(a.y) + row * a.ldy + g * 8, y, sc);
                }
            }
            if (tid == 0)
                a.scales[row] = sc.scale;
        } else {
#pragma unroll
            for (int k = 0; k < kRingGroups; ++k) {
                const int g = k * nt + tid;
                if (g < groups)
                    store_group2<XT>(static_cast<XT *>(a.y) + row * a.ldy + g * 8, s[k]);
            }
        }
    }
    copies_wait<0>();
}

// Whether rows go through the ring, and with how many CTAs per SM: long rows
// (a warp of kRingGroups groups a thread at least) whose ring fits the shared
// memory.
struct RingPlan {
    bool on;
    int block, per_sm;
    size_t smem;
};
RingPlan ring_plan(int64_t D, int64_t row_bytes)
{
    RingPlan p{};
    p.smem = (size_t)kRing * row_bytes;
    p.block = threads_per_row(D, 8, kRingGroups);
    p.on = D >= 1024 && D <= 16384 && p.smem <= 200 << 10;
    p.per_sm = (int)((220 << 10) / (p.smem + 2048));
    const int by_regs = 512 / p.block;
    p.per_sm = p.per_sm < by_regs ? p.per_sm : by_regs;
    p.per_sm = p.per_sm > 8 ? 8 : p.per_sm < 1 ? 1 : p.per_sm;
    return p;
}
template <typename K, typename A>
cudaError_t launch_ring(K kernel, const A &a, const RingPlan &p, int64_t grid, cudaStream_t stream)
{
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 << 10);
    if (e != cudaSuccess)
        return e;
    return launch_k(kernel, dim3((unsigned)grid), dim3(p.block), p.smem, stream, true, a);
}

// Rows off the 16-byte boundaries, one per CTA at a time.  In memory they are
// taken in the 16-byte units of their addresses, through shared memory where
// they keep their shift, with single elements at both ends; between, a thread
// has columns tid, tid + nt, ... of every row, whatever the shifts of the
// arrays.  The units come asynchronously, two rows ahead, the single elements
// in a register, one row ahead.  bf16, us, element by element from memory / so:
// x + residual 16384 x 1003 59 / 37, 8192 x 4095 185 / 62; in 8 bits (x alone)
// 69 / 32, 221 / 62; backward 76 / 48, 197 / 89.  Columns per thread: 16 from 512
// columns on (8192 x 4095 x + residual 62 us, 82 with 8), 8 for shorter rows
// (65536 x 130 41 us, 47 with 16) and for 8 bits, whose second reduction wants
// the warps (with a residual 93 us, 95 with 16; without one 62 and 58).
template <typename T>
struct RowCut {
    static constexpr int VE = 16 / sizeof(T);
    int shift, head, units, tail;
    __device__ __forceinline__ RowCut(const T *p, int D)
    {
        shift = (int)((uintptr_t)p & 15);
        head = shift ? (16 - shift) / (int)sizeof(T) : 0;
        head = head < D ? head : D;
        units = (D - head) / VE;
        tail = D - head - units * VE;
    }
    // The single element of this thread, or -1.
    __device__ __forceinline__ int edge(int D) const
    {
        const int t = threadIdx.x;
        return t < head ? t : t < head + tail ? D - tail + (t - head) : -1;
    }
    __device__ __forceinline__ int at(int col) const { return shift + col * (int)sizeof(T); }
};
template <typename T>
__host__ __device__ constexpr int shifted_bytes(int D)
{
    return (D * (int)sizeof(T) + 15) / 16 * 16 + 16;
}
template <typename T>
__device__ __forceinline__ void shifted_fetch(unsigned char *to, const T *row, int D)
{
    const RowCut<T> c(row, D);
    for (int u = threadIdx.x; u < c.units; u += blockDim.x)
        copy16(to + c.at(c.head) + u * 16, row + c.head + u * RowCut<T>::VE);
}
template <typename T>
__device__ __forceinline__ T shifted_edge(const T *row, int D, bool on)
{
    const int e = on ? RowCut<T>(row, D).edge(D) : -1;
    return e >= 0 ? row[e] : T{};
}
template <typename T>
__device__ __forceinline__ void shifted_put_edge(unsigned char *to, const T *row, int D, T v)
{
    const RowCut<T> c(row, D);
    const int e = c.edge(D);
    if (e >= 0)
        *reinterpret_cast<T *>(to + c.at(e)) = v;
}
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(bf16_t v) { return __uint_as_float((unsigned)v.u << 16); }
__device__ __forceinline__ void from_float(float &o, float v) { o = v; }
__device__ __forceinline__ void from_float(bf16_t &o, float v) { o.u = dev::f2bf(v); }
// A finished row from shared memory to where it belongs.
template <typename T>
__device__ __forceinline__ void shifted_store(T *row, const unsigned char *from, int D)
{
    const RowCut<T> c(row, D);
    for (int u = threadIdx.x; u < c.units; u += blockDim.x)
        *reinterpret_cast<uint4 *>(row + c.head + u * RowCut<T>::VE) =
            *reinterpret_cast<const uint4 *>(from + c.at(c.head) + u * 16);
    const int e = c.edge(D);
    if (e >= 0)
        row[e] = *reinterpret_cast<const T *>(from + c.at(e));
}

template <typename XT, typename RT, bool RES, bool NORM, int OUT, int NV>
__global__ void __launch_bounds__(NV == 16 ? 512 : 1024, 1) k_rmsnorm_shifted(NormArgs a)
{
    using YT = std::conditional_t<OUT == kOutInt, int8_t, XT>;
    extern __shared__ __align__(128) unsigned char sm[];  // [stage][x, residual], h, y
    __shared__ float part[2][2][32];
    const int tid = threadIdx.x, nt = blockDim.x, D = a.D;
    const int x_bytes = shifted_bytes<XT>(D), stage_bytes = x_bytes + (RES ? shifted_bytes<RT>(D) : 0);
    unsigned char *hbuf = sm + kRing * stage_bytes, *ybuf = hbuf + (RES ? shifted_bytes<RT>(D) : 0);
    const XT *x = static_cast<const XT *>(a.x);
    const RT *res = static_cast<const RT *>(a.res);
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    auto fetch = [&](int64_t row, int stage) {
        if (row < a.T) {
            shifted_fetch<XT>(sm + stage * stage_bytes, x + row * a.ldx, D);
            if constexpr (RES)
                shifted_fetch<RT>(sm + stage * stage_bytes + x_bytes, res + row * a.ldr, D);
        }
        copies_commit();
    };
#pragma unroll
    for (int s = 0; s < kRing; ++s)
        fetch(blockIdx.x + (int64_t)s * gridDim.x, s);
    XT xe = shifted_edge<XT>(x + blockIdx.x * a.ldx, D, true);
    RT re{};
    if constexpr (RES)
        re = shifted_edge<RT>(res + blockIdx.x * a.ldr, D, true);
    float g[NV];
    if constexpr (NORM) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float one[1] = {0.f};
            if (k * nt + tid < D)
                load_gain<1>(a.gain, a.gbf16, k * nt + tid, one);
            g[k] = one[0];
        }
    }
    int stage = 0, par = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, par ^= 1) {
        unsigned char *xb = sm + stage * stage_bytes, *rb = xb + x_bytes;
        const XT *xr = x + row * a.ldx;
        const RT *rr = RES ? res + row * a.ldr : nullptr;
        copies_wait<kRing - 1>();
        shifted_put_edge<XT>(xb, xr, D, xe);
        const bool more = row + gridDim.x < a.T;
        xe = shifted_edge<XT>(xr + (int64_t)gridDim.x * a.ldx, D, more);
        if constexpr (RES) {
            shifted_put_edge<RT>(rb, rr, D, re);
            re = shifted_edge<RT>(rr + (int64_t)gridDim.x * a.ldr, D, more);
        }
        __syncthreads();
        RT *hrow = RES ? static_cast<RT *>(a.h) + row * a.ldh : nullptr;
        YT *yrow = static_cast<YT *>(a.y) + row * a.ldy;
        const int xs = (int)((uintptr_t)xr & 15), rs = (int)((uintptr_t)rr & 15), hs = (int)((uintptr_t)hrow & 15),
                  ys = (int)((uintptr_t)yrow & 15);
        float s[NV];
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int j = k * nt + tid;
            s[k] = 0.f;
            if (j < D) {
                s[k] = as_float(reinterpret_cast<const XT *>(xb + xs)[j]);
                if constexpr (RES) {
                    s[k] += as_float(reinterpret_cast<const RT *>(rb + rs)[j]);
                    from_float(reinterpret_cast<RT *>(hbuf + hs)[j], s[k]);
                }
                ss = fmaf(s[k], s[k], ss);
            }
        }
        if constexpr (NORM) {
            const float rstd = 1.f / sqrtf(cta_join<false>(ss, part[par][0]) / (float)D + a.eps);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                s[k] = s[k] * rstd * g[k];
        }
        if constexpr (OUT == kOutInt) {
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                top = max_nan(top, fabsf(s[k]));
            const RowScale sc = row_scale(cta_join<true>(top, part[par][1]));
            unsigned q[NV];
            quants<NV>(s, sc, q);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (k * nt + tid < D)
                    reinterpret_cast<int8_t *>(ybuf + ys)[k * nt + tid] = (int8_t)(q[k] & 0xff);
            if (tid == 0)
                a.scales[row] = sc.scale;
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (k * nt + tid < D)
                    from_float(reinterpret_cast<XT *>(ybuf + ys)[k * nt + tid], s[k]);
        }
        __syncthreads();  // the outputs are whole, and every thread has read its inputs
        fetch(row + (int64_t)kRing * gridDim.x, stage);
        stage = stage + 1 == kRing ? 0 : stage + 1;
        if constexpr (RES)
            shifted_store<RT>(hrow, hbuf, D);
        shifted_store<YT>(yrow, ybuf, D);
    }
    copies_wait<0>();
}

// Columns per thread, threads, CTAs and shared memory of the kernels for
// shifted rows.
struct ShiftPlan {
    bool on;
    int cols, block, per_sm;
    size_t smem;
};
ShiftPlan shift_plan(int64_t D, size_t stage_bytes, size_t out_bytes, bool wide)
{
    ShiftPlan p{};
    p.cols = wide && D >= 512 ? 16 : 8;
    p.block = round32((int)((D + p.cols - 1) / p.cols));
    p.smem = kRing * stage_bytes + out_bytes;
    p.on = D <= 8192 && p.smem <= 200 << 10;
    p.per_sm = (int)((220 << 10) / (p.smem + 2048));
    const int by_regs = (p.cols == 16 ? 768 : 1024) / p.block;
    p.per_sm = p.per_sm < by_regs ? p.per_sm : by_regs;
    p.per_sm = p.per_sm > 32 ? 32 : p.per_sm < 1 ? 1 : p.per_sm;
    return p;
}
template <typename K, typename A>
cudaError_t launch_shifted(K kernel, const A &a, const ShiftPlan &p, int64_t grid, cudaStream_t stream)
{
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 << 10);
    if (e != cudaSuccess)
        return e;
    return launch_k(kernel, dim3((unsigned)grid), dim3(p.block), p.smem, stream, true, a);
}

// Groups per thread: one while the rows alone do not fill the GPU (a call of
// a few tokens is all latency), four otherwise: two or eight were 10 to 60 %
// slower on 65536 x 1024 to 8192 x 8192.  Rows off the 16-byte boundaries go
// through shared memory with their shifts (k_rmsnorm_shifted); those of more than
// 8192 columns, or too wide for it, are taken element by element from memory.
//   The ring where it pays, us, ring / one row at a time:
//   x alone in its type     8192 x 8192 bf16 46 / 49, 16384 x 4096 46 / 46,
//                           65536 x 1024 47 / 42;
//   x + residual            8192 x 8192 88 / 79: the simple form is at the copy
//                           bandwidth already;
//   8 bits of x + residual  all bf16 8000 x 12288 105 / 131, 2048 x 8192 20.5 /
//                           24.0, 4095 x 8192 41.1 / 42.4, but 6000 x 8192 60.7 /
//                           59.1 and 16384 x 4096 82.8 / 74.6; with a residual
//                           in fp32 8192 x 8192 128 / 110, 8000 x 12288 184 / 169.
//   Rows without a norm need few registers: six CTAs of 256 threads per SM (40
// us for 8192 x 8192 bf16, 41 with four).
template <typename XT, typename RT, bool RES, bool NORM, int OUT>
cudaError_t pick_norm(const NormArgs &a, bool grouped8, cudaStream_t stream)
{
    if (grouped8) {
        if (a.T <= kSms && a.D <= 8192)
            return go_norm<XT, RT, RES, NORM, OUT, 8, 1>(a, stream);
        if constexpr (!NORM) {
            if (a.D <= 8192)
                return go_norm<XT, RT, RES, NORM, OUT, 8, 4, 256, 6>(a, stream);
        } else if constexpr (!RES || (OUT == kOutInt && sizeof(RT) == 2)) {
            const RingPlan p = ring_plan(a.D, a.D * (int64_t)(sizeof(XT) + (RES ? sizeof(RT) : 0)));
            const int64_t grid = (int64_t)kSms * p.per_sm;
            const bool pays = !RES ? a.D > (OUT == kOutInt ? 1024 : 4096)
                                   : a.D > 8192 || (a.D > 4096 && a.T <= 14 * grid);
            if (p.on && pays && a.T >= 2 * grid)
                return p.block <= 256
                           ? launch_ring(k_rmsnorm_ring<XT, RT, RES, OUT, 256, 2>, a, p, grid, stream)
                           : launch_ring(k_rmsnorm_ring<XT, RT, RES, OUT, 512, 1>, a, p, grid, stream);
        }
        return go_norm<XT, RT, RES, NORM, OUT, 8, 4>(a, stream);
    }
    using YT = std::conditional_t<OUT == kOutInt, int8_t, XT>;
    const size_t r = RES ? shifted_bytes<RT>(a.D) : 0;
    const ShiftPlan p = shift_plan(a.D, shifted_bytes<XT>(a.D) + r, r + shifted_bytes<YT>(a.D), OUT == kOutSame);
    if (!p.on)
        return go_norm<XT, RT, RES, NORM, OUT, 1, 32>(a, stream);
    const int64_t most = (int64_t)kSms * p.per_sm, grid = a.T < most ? a.T : most;
    if constexpr (OUT == kOutSame) {
        if (p.cols == 16)
            return launch_shifted(k_rmsnorm_shifted<XT, RT, RES, NORM, OUT, 16>, a, p, grid, stream);
    }
    return launch_shifted(k_rmsnorm_shifted<XT, RT, RES, NORM, OUT, 8>, a, p, grid, stream);
}

template <int OUT>
cudaError_t launch_norm(const NormArgs &a, int xtype, int rtype, bool grouped8, cudaStream_t stream)
{
    const bool xb = xtype == EMBER_BF16, rb = rtype == EMBER_BF16;
    if (a.res == nullptr)
        return xb ? pick_norm<bf16_t, bf16_t, false, true, OUT>(a, grouped8, stream)
                  : pick_norm<float, float, false, true, OUT>(a, grouped8, stream);
    if (xb)
        return rb ? pick_norm<bf16_t, bf16_t, true, true, OUT>(a, grouped8, stream)
                  : pick_norm<bf16_t, float, true, true, OUT>(a, grouped8, stream);
    return rb ? pick_norm<float, bf16_t, true, true, OUT>(a, grouped8, stream)
              : pick_norm<float, float, true, true, OUT>(a, grouped8, stream);
}

// ---------------------------------------------------------------------------
// Gradients.  A persistent CTA takes rows b, b + gridDim, ...; a thread keeps
// the same columns in every row, so that the sums of dgain stay in its
// registers; at the end each row group writes them as one row of `partial`,
// and a second kernel adds the rows in order.  The grid depends on the sizes,
// types and alignment only, and with it every bit of dgain.
// ---------------------------------------------------------------------------
struct BackArgs {
    const void *dy, *h, *dres, *gain;
    void *dx;
    float *partial;  // [gridDim * rows per CTA][D]
    int64_t lddy, ldh, lddres, lddx, T;
    int D, tpr, gbf16;
    float eps;
};

template <typename XT, bool RES, int VEC, int NV, int MAXT>
__global__ void __launch_bounds__(MAXT, 1) k_rmsnorm_back(BackArgs a)
{
    __shared__ float part[2][2][32];  // by parity of the row: one barrier per row
    const int rpc = blockDim.x / a.tpr;
    const int group = threadIdx.x / a.tpr;
    const int lane = threadIdx.x % a.tpr;
    const int w = threadIdx.x >> 5;
    const int nw = a.tpr >> 5;
    const int w0 = w / nw * nw;
    dev::grid_dep_wait();
    dev::grid_dep_launch();

    float acc[NV][VEC];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            acc[k][e] = 0.f;
    const float inv_D = 1.f / (float)a.D;
    int par = 0;
    for (int64_t base = (int64_t)blockIdx.x * rpc; base < a.T; base += (int64_t)gridDim.x * rpc, par ^= 1) {
        const int64_t row = base + group;
        const bool live = row < a.T;
        Raw<XT, VEC> dy[NV], h[NV], dr[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int col = (k * a.tpr + lane) * VEC;
            const bool on = live && col < a.D;
            dy[k] = on ? load_raw<XT, VEC>(static_cast<const XT *>(a.dy) + row * a.lddy + col) : zero_raw<XT, VEC>();
            h[k] = on ? load_raw<XT, VEC>(static_cast<const XT *>(a.h) + row * a.ldh + col) : zero_raw<XT, VEC>();
            if constexpr (RES)
                dr[k] = on ? load_raw<XT, VEC>(static_cast<const XT *>(a.dres) + row * a.lddres + col)
                           : zero_raw<XT, VEC>();
        }
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int col = (k * a.tpr + lane) * VEC;
            if (col < a.D) {
                float g[VEC], fy[VEC], fh[VEC];
                load_gain<VEC>(a.gain, a.gbf16, col, g);
                unpack<XT, VEC>(dy[k], fy);
                unpack<XT, VEC>(h[k], fh);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    ss = fmaf(fh[e], fh[e], ss);
                    dot = fmaf(fy[e] * g[e], fh[e], dot);
                }
            }
        }
        ss = warp_sum(ss);
        dot = warp_sum(dot);
        if (nw > 1) {
            if ((threadIdx.x & 31) == 0) {
                part[par][0][w] = ss;
                part[par][1][w] = dot;
            }
            __syncthreads();
            ss = part[par][0][w0];
            dot = part[par][1][w0];
            for (int k = 1; k < nw; ++k) {
                ss += part[par][0][w0 + k];
                dot += part[par][1][w0 + k];
            }
        }
        const float r = 1.f / sqrtf(ss * inv_D + a.eps);
        const float c = r * r * (dot * inv_D);
        if (!live)
            continue;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int col = (k * a.tpr + lane) * VEC;
            if (col < a.D) {
                float g[VEC], fy[VEC], fh[VEC], o[VEC];
                load_gain<VEC>(a.gain, a.gbf16, col, g);
                unpack<XT, VEC>(dy[k], fy);
                unpack<XT, VEC>(h[k], fh);
                if constexpr (RES)
                    unpack<XT, VEC>(dr[k], o);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float v = r * fmaf(-fh[e], c, fy[e] * g[e]);
                    o[e] = RES ? v + o[e] : v;
                    acc[k][e] = fmaf(fy[e], fh[e] * r, acc[k][e]);
                }
                store_group<XT, VEC>(static_cast<XT *>(a.dx) + row * a.lddx + col, o);
            }
        }
    }
    float *p = a.partial + ((int64_t)blockIdx.x * rpc + group) * a.D;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int col = (k * a.tpr + lane) * VEC;
        if (col < a.D) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                p[col + e] = acc[k][e];
        }
    }
}

// The same for long rows of whole groups, through the ring of k_rmsnorm_ring.
template <typename XT, bool RES, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) k_rmsnorm_back_ring(BackArgs a)
{
    constexpr int NIN = RES ? 3 : 2;
    extern __shared__ __align__(128) unsigned char ring[];  // [stage][dy, h, dres]
    __shared__ float part[2][2][32];
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, w = tid >> 5, nw = nt >> 5;
    const int groups = a.D / 8;
    const int row_bytes = a.D * (int)sizeof(XT);
    dev::grid_dep_wait();
    dev::grid_dep_launch();

    auto fetch = [&](int64_t row, int stage) {
        if (row < a.T) {
            unsigned char *to = ring + (size_t)stage * NIN * row_bytes;
            ring_fetch<XT>(to, static_cast<const XT *>(a.dy) + row * a.lddy, groups);
            ring_fetch<XT>(to + row_bytes, static_cast<const XT *>(a.h) + row * a.ldh, groups);
            if constexpr (RES)
                ring_fetch<XT>(to + 2 * row_bytes, static_cast<const XT *>(a.dres) + row * a.lddres, groups);
        }
        copies_commit();
    };
#pragma unroll
    for (int s = 0; s < kRing; ++s)
        fetch(blockIdx.x + (int64_t)s * gridDim.x, s);
    f2 acc[kRingGroups][4], ga[kRingGroups][4];
    gains2(a.gain, a.gbf16, groups, ga);
#pragma unroll
    for (int k = 0; k < kRingGroups; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            acc[k][q] = make2(0.f, 0.f);
    const float inv_D = 1.f / (float)a.D;
    int stage = 0, par = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, par ^= 1) {
        copies_wait<kRing - 1>();
        const unsigned char *from = ring + (size_t)stage * NIN * row_bytes;
        f2 ss2 = make2(0.f, 0.f), dot2 = make2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kRingGroups; ++k) {
            const int g = k * nt + tid;
            if (g < groups) {
                f2 fy[4], fh[4];
                ring_read<XT>(from, g, fy);
                ring_read<XT>(from + row_bytes, g, fh);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    ss2 = fma2(fh[q], fh[q], ss2);
                    dot2 = fma2(mul2(fy[q], ga[k][q]), fh[q], dot2);
                }
            }
        }
        float ss = warp_sum(sum2(ss2)), dot = warp_sum(sum2(dot2));
        if (nw > 1) {
            if (lane == 0) {
                part[par][0][w] = ss;
                part[par][1][w] = dot;
            }
            __syncthreads();
            ss = warp_sum(lane < nw ? part[par][0][lane] : 0.f);
            dot = warp_sum(lane < nw ? part[par][1][lane] : 0.f);
        }
        const float r = 1.f / sqrtf(ss * inv_D + a.eps);
        const float c = r * r * (dot * inv_D);
        const f2 r2 = make2(r, r), mc2 = make2(-c, -c);
#pragma unroll
        for (int k = 0; k < kRingGroups; ++k) {
            const int g = k * nt + tid;
            if (g < groups) {
                f2 fy[4], fh[4], o[4];
                ring_read<XT>(from, g, fy);
                ring_read<XT>(from + row_bytes, g, fh);
                if constexpr (RES)
                    ring_read<XT>(from + 2 * row_bytes, g, o);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f2 v = fma2(fh[q], mc2, mul2(fy[q], ga[k][q]));
                    o[q] = RES ? fma2(v, r2, o[q]) : mul2(v, r2);
                    acc[k][q] = fma2(fy[q], mul2(fh[q], r2), acc[k][q]);
                }
                store_group2<XT>(static_cast<XT *>(a.dx) + row * a.lddx + g * 8, o);
            }
        }
        fetch(row + (int64_t)kRing * gridDim.x, stage);
        stage = stage + 1 == kRing ? 0 : stage + 1;
    }
    copies_wait<0>();
    float *p = a.partial + (int64_t)blockIdx.x * a.D;
#pragma unroll
    for (int k = 0; k < kRingGroups; ++k) {
        const int g = k * nt + tid;
        if (g < groups)
            store_group2<float>(p + g * 8, acc[k]);
    }
}

// The same for rows off the 16-byte boundaries, as k_rmsnorm_shifted takes them.
template <typename XT, bool RES, int NV>
__global__ void __launch_bounds__(NV == 16 ? 512 : 1024, 1) k_rmsnorm_back_shifted(BackArgs a)
{
    constexpr int NIN = RES ? 3 : 2;
    extern __shared__ __align__(128) unsigned char sm[];  // [stage][dy, h, dres], dx
    __shared__ float part[2][2][32];
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, w = tid >> 5, nw = nt >> 5, D = a.D;
    const int row_bytes = shifted_bytes<XT>(D), stage_bytes = NIN * row_bytes;
    unsigned char *obuf = sm + kRing * stage_bytes;
    const XT *in[3] = {static_cast<const XT *>(a.dy), static_cast<const XT *>(a.h), static_cast<const XT *>(a.dres)};
    const int64_t ld[3] = {a.lddy, a.ldh, a.lddres};
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    auto fetch = [&](int64_t row, int stage) {
        if (row < a.T) {
#pragma unroll
            for (int i = 0; i < NIN; ++i)
                shifted_fetch<XT>(sm + stage * stage_bytes + i * row_bytes, in[i] + row * ld[i], D);
        }
        copies_commit();
    };
#pragma unroll
    for (int s = 0; s < kRing; ++s)
        fetch(blockIdx.x + (int64_t)s * gridDim.x, s);
    XT edge[NIN];
#pragma unroll
    for (int i = 0; i < NIN; ++i)
        edge[i] = shifted_edge<XT>(in[i] + blockIdx.x * ld[i], D, true);
    float g[NV], acc[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        float one[1] = {0.f};
        if (k * nt + tid < D)
            load_gain<1>(a.gain, a.gbf16, k * nt + tid, one);
        g[k] = one[0];
        acc[k] = 0.f;
    }
    const float inv_D = 1.f / (float)D;
    int stage = 0, par = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, par ^= 1) {
        copies_wait<kRing - 1>();
        const bool more = row + gridDim.x < a.T;
        const unsigned char *from[NIN];
#pragma unroll
        for (int i = 0; i < NIN; ++i) {
            unsigned char *b = sm + stage * stage_bytes + i * row_bytes;
            const XT *r = in[i] + row * ld[i];
            shifted_put_edge<XT>(b, r, D, edge[i]);
            edge[i] = shifted_edge<XT>(r + (int64_t)gridDim.x * ld[i], D, more);
            from[i] = b + ((uintptr_t)r & 15);
        }
        __syncthreads();
        float fy[NV], fh[NV], fr[NV];
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int j = k * nt + tid;
            const bool on = j < D;
            fy[k] = on ? as_float(reinterpret_cast<const XT *>(from[0])[j]) : 0.f;
            fh[k] = on ? as_float(reinterpret_cast<const XT *>(from[1])[j]) : 0.f;
            fr[k] = 0.f;
            if constexpr (RES)
                fr[k] = on ? as_float(reinterpret_cast<const XT *>(from[2])[j]) : 0.f;
            ss = fmaf(fh[k], fh[k], ss);
            dot = fmaf(fy[k] * g[k], fh[k], dot);
        }
        ss = warp_sum(ss);
        dot = warp_sum(dot);
        if (nw > 1) {
            if (lane == 0) {
                part[par][0][w] = ss;
                part[par][1][w] = dot;
            }
            __syncthreads();
            ss = warp_sum(lane < nw ? part[par][0][lane] : 0.f);
            dot = warp_sum(lane < nw ? part[par][1][lane] : 0.f);
        }
        const float r = 1.f / sqrtf(ss * inv_D + a.eps);
        const float c = r * r * (dot * inv_D);
        XT *orow = static_cast<XT *>(a.dx) + row * a.lddx;
        XT *o = reinterpret_cast<XT *>(obuf + ((uintptr_t)orow & 15));
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int j = k * nt + tid;
            if (j < D) {
                from_float(o[j], fmaf(r, fmaf(-fh[k], c, fy[k] * g[k]), fr[k]));
                acc[k] = fmaf(fy[k], fh[k] * r, acc[k]);
            }
        }
        __syncthreads();
        fetch(row + (int64_t)kRing * gridDim.x, stage);
        stage = stage + 1 == kRing ? 0 : stage + 1;
        shifted_store<XT>(orow, obuf, D);
    }
    copies_wait<0>();
    float *p = a.partial + (int64_t)blockIdx.x * D;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (k * nt + tid < D)
            p[k * nt + tid] = acc[k];
}

// dgain_j = the sum of the n partial rows of column j: COLS columns a CTA, each
// by 1024 / COLS threads, which take every so-many-th row and are joined in order.
template <int COLS>
__global__ void __launch_bounds__(1024) k_dgain(const float *__restrict__ partial, int n, int D,
                                                float *__restrict__ dgain)
{
    __shared__ float part[32][COLS + 1];
    const int c = threadIdx.x % COLS, r = threadIdx.x / COLS, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int col = blockIdx.x * COLS + c;
    dev::grid_dep_wait();
    float s = 0.f;
    constexpr int R = 1024 / COLS;
    if (col < D)
        for (int k = r; k < n; k += 4 * R) {  // four loads at once
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int q = k + e * R;
                v[e] = partial[(int64_t)(q < n ? q : r) * D + col];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s += k + e * R < n ? v[e] : 0.f;
        }
#pragma unroll
    for (int o = COLS; o < 32; o *= 2)  // the rows of this warp
        s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane < COLS)
        part[warp][c] = s;
    __syncthreads();
    if (warp < COLS && blockIdx.x * COLS + warp < D) {  // warp k joins column k of the block
        s = warp_sum(part[lane][warp]);
        if (lane == 0)
            dgain[blockIdx.x * COLS + warp] = s;
    }
}

// Columns per CTA of k_dgain: fewer where 32 would leave SMs idle and there are
// rows enough to share out.  The backward pass with 32 / 16 / 8, us: 8192 x 256
// fp32 22.6 / 16.5 / 13.8, 2048 x 1024 fp32 9.8 / 8.7 / 8.3, 4096 x 4096 bf16
// 21.0 / 20.1 / 21.0, 2048 x 8192 22.8 / 23.3 / 25.2, 64 x 4096 4.6 / 5.0 / 5.7.
cudaError_t launch_dgain(const float *partial, int n, int D, float *dgain, cudaStream_t stream)
{
    auto go = [&](auto kernel, int cols) {
        return launch_k(kernel, dim3((unsigned)((D + cols - 1) / cols)), dim3(1024), 0, stream, true, partial, n, D, dgain);
    };
    if (n <= 128 || D > 32 * kSms)
        return go(k_dgain<32>, 32);
    return D > 2048 ? go(k_dgain<16>, 16) : go(k_dgain<8>, 8);
}

struct BackPlan {
    RingPlan ring;
    ShiftPlan shift;
    int vec, nv, tpr, block, grid;
    int64_t parts;  // partial rows
};

// Rows of whole groups from 1024 columns on go through the ring where it fits,
// rows off the boundaries through shared memory with their shifts; the rest keeps
// one row in registers: up to 1023 columns, and those too wide for the other two.
BackPlan back_plan(int64_t T, int64_t D, int esize, bool res, bool grouped8)
{
    BackPlan p{};
    p.ring = ring_plan(D, (res ? 3 : 2) * D * esize);
    p.ring.on = p.ring.on && grouped8;
    const size_t row = (size_t)(esize == 2 ? shifted_bytes<bf16_t>((int)D) : shifted_bytes<float>((int)D));
    p.shift = shift_plan(D, (res ? 3 : 2) * row, row, true);
    p.shift.on = p.shift.on && !grouped8;
    p.vec = grouped8 ? 8 : 1;
    p.nv = grouped8 ? (D < 1024 ? 1 : 4) : 32;
    p.tpr = threads_per_row(D, p.vec, p.nv);
    p.block = p.tpr < kMinBlock ? kMinBlock : p.tpr;
    const int64_t rpc = p.ring.on || p.shift.on ? 1 : p.block / p.tpr;
    const int64_t want = (T + rpc - 1) / rpc;
    const int64_t most = (int64_t)kSms * (p.ring.on    ? p.ring.per_sm
                                          : p.shift.on ? p.shift.per_sm
                                                       : (p.block >= 1024 ? 1 : 1024 / p.block));
    p.grid = (int)(want < most ? want : most);
    p.parts = p.grid * rpc;
    return p;
}

template <typename XT, bool RES>
cudaError_t launch_back(BackArgs a, const BackPlan &p, cudaStream_t stream)
{
    a.tpr = p.tpr;
    if (p.ring.on)
        return p.ring.block <= 256 ? launch_ring(k_rmsnorm_back_ring<XT, RES, 256, 2>, a, p.ring, p.grid, stream)
                                   : launch_ring(k_rmsnorm_back_ring<XT, RES, 512, 1>, a, p.ring, p.grid, stream);
    if (p.shift.on)
        return p.shift.cols == 16 ? launch_shifted(k_rmsnorm_back_shifted<XT, RES, 16>, a, p.shift, p.grid, stream)
                                  : launch_shifted(k_rmsnorm_back_shifted<XT, RES, 8>, a, p.shift, p.grid, stream);
    auto go = [&](auto kernel) { return launch_k(kernel, dim3(p.grid), dim3(p.block), 0, stream, true, a); };
    if (p.vec == 8) {
        if (p.nv == 1)
            return go(k_rmsnorm_back<XT, RES, 8, 1, 128>);
        if constexpr (sizeof(XT) == 4) {  // bf16 rows of up to 16384 columns always fit the ring
            if (p.block <= 512)
                return go(k_rmsnorm_back<XT, RES, 8, 4, 512>);
        }
        return go(k_rmsnorm_back<XT, RES, 8, 4, 1024>);
    }
    return p.block <= 512 ? go(k_rmsnorm_back<XT, RES, 1, 32, 512>) : go(k_rmsnorm_back<XT, RES, 1, 32, 1024>);
}

// 8-bit rows back as what they stand for: q scale.  `tpr` threads a row, as
// many rows as fit 256 threads; few rows are cut along their columns too.
template <typename YT, int VEC>
__global__ void __launch_bounds__(256) k_dequantize(const int8_t *__restrict__ q, int64_t ldq,
                                                    const float *__restrict__ scales, int64_t T, int D, int tpr,
                                                    YT *__restrict__ y, int64_t ldy)
{
    const int64_t row = (int64_t)blockIdx.x * (256 / tpr) + threadIdx.x / tpr;
    const int step = gridDim.y * tpr * VEC;
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    if (row >= T)
        return;
    const float s = scales[row];
#pragma unroll 4
    for (int col = (blockIdx.y * tpr + threadIdx.x % tpr) * VEC; col < D; col += step) {
        float f[VEC];
        if constexpr (VEC == 8) {
            const uint2 u = *reinterpret_cast<const uint2 *>(q + row * ldq + col);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                f[e] = (float)(int8_t)((e < 4 ? u.x : u.y) >> (8 * (e & 3))) * s;
        } else
            f[0] = (float)q[row * ldq + col] * s;
        store_group<YT, VEC>(y + row * ldy + col, f);
    }
}

// What every norm has in common; EMBER_OK with nothing to do when T is 0.
ember_status check_rows(const void *p, int64_t ld, int dtype, int64_t T, int64_t D)
{
    if (T > 0 && !p)
        return EMBER_ERR_INVALID_ARG;
    if (T < 0 || D < 1 || ld < D || ld > (int64_t(1) << 40) || (T > 0 && ld > (int64_t(1) << 61) / T))
        return EMBER_ERR_INVALID_ARG;
    if (!dtype_ok(dtype))
        return EMBER_ERR_DTYPE;
    if (T > INT32_MAX || D > kMaxRowCols)
        return EMBER_ERR_UNSUPPORTED;
    if (!aligned(p, elem_size(dtype)))
        return EMBER_ERR_ALIGNMENT;
    return EMBER_OK;
}

#define EMBER_TRY(call)             \
    do {                            \
        const ember_status st_ = (call); \
        if (st_ != EMBER_OK)        \
            return st_;             \
    } while (0)

ember_status norm_common(NormArgs &a, bool &grouped8, const void *x, int64_t ldx, ember_wdtype xtype,
                         const void *residual, int64_t ldr, ember_wdtype rtype, const void *gain,
                         ember_wdtype gtype, int64_t T, int64_t D, float eps, void *h, int64_t ldh)
{
    if (!(eps >= 0.f) || eps > 3.4e38f || (residual == nullptr) != (h == nullptr))
        return EMBER_ERR_INVALID_ARG;
    EMBER_TRY(check_rows(x, ldx, xtype, T, D));
    if (residual) {
        EMBER_TRY(check_rows(residual, ldr, rtype, T, D));
        EMBER_TRY(check_rows(h, ldh, rtype, T, D));
    }
    if (gain && !dtype_ok(gtype))
        return EMBER_ERR_DTYPE;
    if (gain && !aligned(gain, elem_size(gtype)))
        return EMBER_ERR_ALIGNMENT;
    a.x = x;
    a.res = residual;
    a.gain = gain;
    a.h = h;
    a.ldx = ldx;
    a.ldr = ldr;
    a.ldh = ldh;
    a.T = T;
    a.D = (int)D;
    a.gbf16 = gtype == EMBER_BF16;
    a.eps = eps;
    grouped8 = D % 8 == 0 && grouped(x, ldx, xtype) && grouped(residual, ldr, rtype) && grouped(h, ldh, rtype) &&
               aligned(gain, 8 * elem_size(gtype));
    return EMBER_OK;
}

}  // namespace
}  // namespace ember

using namespace ember;

extern "C" {

ember_status ember_rmsnorm(const void *x, int64_t ldx, ember_wdtype xtype, const void *residual, int64_t ldr,
                           ember_wdtype rtype, const void *gain, ember_wdtype gtype, int64_t T, int64_t D, float eps,
                           void *h, int64_t ldh, void *y, int64_t ldy, void *stream)
{
    NormArgs a{};
    bool grouped8;
    EMBER_TRY(norm_common(a, grouped8, x, ldx, xtype, residual, ldr, rtype, gain, gtype, T, D, eps, h, ldh));
    EMBER_TRY(check_rows(y, ldy, xtype, T, D));
    if (T == 0)
        return EMBER_OK;
    a.y = y;
    a.ldy = ldy;
    grouped8 = grouped8 && grouped(y, ldy, xtype);
    return launched(launch_norm<kOutSame>(a, xtype, rtype, grouped8, (cudaStream_t)stream));
}

ember_status ember_rmsnorm_quant(const void *x, int64_t ldx, ember_wdtype xtype, const void *residual, int64_t ldr,
                                 ember_wdtype rtype, const void *gain, ember_wdtype gtype, int64_t T, int64_t D,
                                 float eps, void *h, int64_t ldh, int8_t *q, int64_t ldq, float *scales, void *stream)
{
    NormArgs a{};
    bool grouped8;
    EMBER_TRY(norm_common(a, grouped8, x, ldx, xtype, residual, ldr, rtype, gain, gtype, T, D, eps, h, ldh));
    if (ldq < D || (T > 0 && (!q || !scales)))
        return EMBER_ERR_INVALID_ARG;
    if (!aligned(scales, 4))
        return EMBER_ERR_ALIGNMENT;
    if (T == 0)
        return EMBER_OK;
    a.y = q;
    a.ldy = ldq;
    a.scales = scales;
    grouped8 = grouped8 && aligned(q, 8) && ldq % 8 == 0;
    return launched(launch_norm<kOutInt>(a, xtype, rtype, grouped8, (cudaStream_t)stream));
}

ember_status ember_quantize_rows(const void *x, int64_t ldx, ember_wdtype xtype, int64_t T, int64_t D, int8_t *q,
                                 int64_t ldq, float *scales, void *stream)
{
    EMBER_TRY(check_rows(x, ldx, xtype, T, D));
    if (ldq < D || (T > 0 && (!q || !scales)))
        return EMBER_ERR_INVALID_ARG;
    if (!aligned(scales, 4))
        return EMBER_ERR_ALIGNMENT;
    if (T == 0)
        return EMBER_OK;
    NormArgs a{};
    a.x = x;
    a.ldx = ldx;
    a.T = T;
    a.D = (int)D;
    a.y = q;
    a.ldy = ldq;
    a.scales = scales;
    const bool grouped8 = D % 8 == 0 && grouped(x, ldx, xtype) && aligned(q, 8) && ldq % 8 == 0;
    return launched(xtype == EMBER_BF16
                        ? pick_norm<bf16_t, bf16_t, false, false, kOutInt>(a, grouped8, (cudaStream_t)stream)
                        : pick_norm<float, float, false, false, kOutInt>(a, grouped8, (cudaStream_t)stream));
}

ember_status ember_dequantize_rows(const int8_t *q, int64_t ldq, const float *scales, int64_t T, int64_t D, void *y,
                                   int64_t ldy, ember_wdtype ytype, void *stream)
{
    EMBER_TRY(check_rows(y, ldy, ytype, T, D));
    if (ldq < D || (T > 0 && (!q || !scales)))
        return EMBER_ERR_INVALID_ARG;
    if (!aligned(scales, 4))
        return EMBER_ERR_ALIGNMENT;
    if (T == 0)
        return EMBER_OK;
    const bool grouped8 = D % 8 == 0 && aligned(q, 8) && ldq % 8 == 0 && grouped(y, ldy, ytype);
    // four groups a thread in a long call, one otherwise
    const int64_t groups = grouped8 ? D / 8 : D, per = T <= kSms ? 1 : 4;
    int tpr = 32;
    while (tpr < 256 && tpr * per < groups)
        tpr *= 2;
    const int64_t rpc = 256 / tpr, cols = T <= kSms ? (groups + tpr - 1) / tpr : 1;
    const dim3 grid((unsigned)((T + rpc - 1) / rpc), (unsigned)cols);
    auto go = [&](auto kernel, auto *yt) {
        return launch_k(kernel, grid, dim3(256), 0, (cudaStream_t)stream, true, q, ldq, scales, T, (int)D, tpr, yt, ldy);
    };
    if (ytype == EMBER_BF16)
        return launched(grouped8 ? go(k_dequantize<bf16_t, 8>, static_cast<bf16_t *>(y))
                                 : go(k_dequantize<bf16_t, 1>, static_cast<bf16_t *>(y)));
    return launched(grouped8 ? go(k_dequantize<float, 8>, static_cast<float *>(y))
                             : go(k_dequantize<float, 1>, static_cast<float *>(y)));
}

size_t ember_rmsnorm_backward_workspace_bytes(int64_t T, int64_t D)
{
    if (T < 0 || D < 1 || T > INT32_MAX || D > kMaxRowCols)
        return 0;
    int64_t most = 0;
    for (int k = 0; k < 8; ++k) {  // whatever the types, the alignment and dres
        const int64_t n = back_plan(T, D, k & 1 ? 4 : 2, k & 2, k & 4).parts;
        most = most > n ? most : n;
    }
    return sizeof(float) * (size_t)(most * D);
}

ember_status ember_rmsnorm_backward(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *dres,
                                    int64_t lddres, ember_wdtype type, const void *gain, ember_wdtype gtype, int64_t T,
                                    int64_t D, float eps, void *dx, int64_t lddx, float *dgain, void *workspace,
                                    size_t bytes, void *stream)
{
    if (!(eps >= 0.f) || eps > 3.4e38f || !dgain)
        return EMBER_ERR_INVALID_ARG;
    EMBER_TRY(check_rows(dy, lddy, type, T, D));
    EMBER_TRY(check_rows(h, ldh, type, T, D));
    EMBER_TRY(check_rows(dx, lddx, type, T, D));
    if (dres)
        EMBER_TRY(check_rows(dres, lddres, type, T, D));
    if (gain && !dtype_ok(gtype))
        return EMBER_ERR_DTYPE;
    if ((gain && !aligned(gain, elem_size(gtype))) || !aligned(dgain, 4) || !aligned(workspace, 16))
        return EMBER_ERR_ALIGNMENT;
    if (T == 0)  // no rows: the sums are zero
        return launched(cudaMemsetAsync(dgain, 0, sizeof(float) * (size_t)D, (cudaStream_t)stream));
    const bool grouped8 = D % 8 == 0 && grouped(dy, lddy, type) && grouped(h, ldh, type) &&
                          grouped(dres, lddres, type) && grouped(dx, lddx, type) && aligned(gain, 8 * elem_size(gtype));
    const BackPlan p = back_plan(T, D, (int)elem_size(type), dres != nullptr, grouped8);
    if (!workspace || bytes < sizeof(float) * (size_t)(p.parts * D))
        return EMBER_ERR_WORKSPACE;
    BackArgs a{};
    a.dy = dy;
    a.h = h;
    a.dres = dres;
    a.gain = gain;
    a.dx = dx;
    a.partial = static_cast<float *>(workspace);
    a.lddy = lddy;
    a.ldh = ldh;
    a.lddres = lddres;
    a.lddx = lddx;
    a.T = T;
    a.D = (int)D;
    a.gbf16 = gtype == EMBER_BF16;
    a.eps = eps;
    const cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e;
    if (type == EMBER_BF16)
        e = dres ? launch_back<bf16_t, true>(a, p, s) : launch_back<bf16_t, false>(a, p, s);
    else
        e = dres ? launch_back<float, true>(a, p, s) : launch_back<float, false>(a, p, s);
    if (e == cudaSuccess)
        e = launch_dgain(a.partial, (int)p.parts, (int)D, dgain, s);
    return launched(e);
}

}  // extern "C"
