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

// q = y / scale rounded to nearest even, |q| <= 127.  A row of zeros has the
// scale 0 and zeros; a row with an infinity or a NaN has the scale NaN and
// zeros, so that what is formed from it is NaN throughout.
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
    } else if (s.scale >= 1e-30f) {
        s.inv = 1.f / s.scale;
    } else if (s.scale > 0.f) {  // 1 / scale may overflow, and scale itself be subnormal
        s.divide = true;
    }
    return s;
}
__device__ __forceinline__ int quant(float y, const RowScale &s)
{
    if (s.divide)
        return max(-127, min(127, __float2int_rn(y / s.scale)));
    if (s.inv == 0.f)
        return 0;
    return max(-127, min(127, __float2int_rn(y * s.inv)));
}

template <int VEC>
__device__ __forceinline__ void store_q(int8_t *p, const float (&y)[VEC], const RowScale &s)
{
    if constexpr (VEC == 8) {
        unsigned u[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            u[e >> 2] |= (unsigned)(quant(y[e], s) & 0xff) << (8 * (e & 3));
        *reinterpret_cast<uint2 *>(p) = make_uint2(u[0], u[1]);
    } else
        *p = (int8_t)quant(y[0], s);
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
template <typename XT, typename RT, bool RES, bool NORM, int OUT, int VEC, int NV>
__global__ void __launch_bounds__(1024) k_rmsnorm(NormArgs a)
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

template <typename XT, typename RT, bool RES, bool NORM, int OUT, int VEC, int NV>
cudaError_t go_norm(NormArgs a, cudaStream_t stream)
{
    a.tpr = threads_per_row(a.D, VEC, NV);
    const int block = a.tpr < kMinBlock ? kMinBlock : a.tpr;
    const int64_t rpc = block / a.tpr;
    return launch_k(k_rmsnorm<XT, RT, RES, NORM, OUT, VEC, NV>, dim3((unsigned)((a.T + rpc - 1) / rpc)),
                    dim3(block), 0, stream, true, a);
}

// Groups per thread: one while the rows alone do not fill the GPU (a call of
// a few tokens is all latency), four otherwise (more loads in flight per
// thread, fewer warps to join); rows off the 16-byte boundaries are taken
// element by element.
template <typename XT, typename RT, bool RES, bool NORM, int OUT>
cudaError_t pick_norm(const NormArgs &a, bool grouped8, cudaStream_t stream)
{
    if (grouped8) {
        if (a.T <= kSms && a.D <= 8192)
            return go_norm<XT, RT, RES, NORM, OUT, 8, 1>(a, stream);
        return go_norm<XT, RT, RES, NORM, OUT, 8, 4>(a, stream);
    }
    if (a.D <= 4096)
        return go_norm<XT, RT, RES, NORM, OUT, 1, 4>(a, stream);
    return go_norm<XT, RT, RES, NORM, OUT, 1, 32>(a, stream);
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
// and a second kernel adds the rows in order.  The grid depends on (T, D)
// only, and with it every bit of dgain.
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
__global__ void __launch_bounds__(MAXT) k_rmsnorm_back(BackArgs a)
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

// The same for long rows of whole groups, one row per CTA at a time.  The rows
// of dy, h and dres come through a ring of two rows in shared memory, filled by
// asynchronous copies; a thread copies what it will read itself, so the ring
// needs no barrier, and the next two rows are on their way while one is
// reduced and written.
constexpr int kBackStages = 2;

__device__ __forceinline__ void copy16(void *smem, const void *p)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(p)
                 : "memory");
}

template <typename XT, bool RES, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) k_rmsnorm_back_ring(BackArgs a)
{
    constexpr int NV = 4;                   // groups of 8 per thread
    constexpr int GB = 8 * sizeof(XT);      // bytes of a group
    constexpr int NIN = RES ? 3 : 2;
    extern __shared__ __align__(128) unsigned char ring[];  // [stage][input][group of the row]
    __shared__ float part[2][2][32];
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, w = tid >> 5, nw = nt >> 5;
    const int groups = a.D / 8;
    const int row_bytes = a.D * (int)sizeof(XT);
    dev::grid_dep_wait();
    dev::grid_dep_launch();

    auto fetch = [&](int64_t row, int stage) {
        if (row < a.T) {
            const unsigned char *in[3] = {
                reinterpret_cast<const unsigned char *>(static_cast<const XT *>(a.dy) + row * a.lddy),
                reinterpret_cast<const unsigned char *>(static_cast<const XT *>(a.h) + row * a.ldh),
                RES ? reinterpret_cast<const unsigned char *>(static_cast<const XT *>(a.dres) + row * a.lddres)
                    : nullptr};
#pragma unroll
            for (int i = 0; i < NIN; ++i) {
                unsigned char *to = ring + (size_t)(stage * NIN + i) * row_bytes;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const int g = k * nt + tid;
                    if (g < groups) {
#pragma unroll
                        for (int b = 0; b < GB; b += 16)
                            copy16(to + g * GB + b, in[i] + g * GB + b);
                    }
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto held = [&](int stage, int i, int g) {
        const unsigned char *p = ring + (size_t)(stage * NIN + i) * row_bytes + g * GB;
        Raw<XT, 8> r;
        if constexpr (sizeof(XT) == 2)
            r.v = *reinterpret_cast<const uint4 *>(p);
        else {
            r.a = reinterpret_cast<const float4 *>(p)[0];
            r.b = reinterpret_cast<const float4 *>(p)[1];
        }
        return r;
    };

    float acc[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            acc[k][e] = 0.f;
    const float inv_D = 1.f / (float)a.D;
#pragma unroll
    for (int s = 0; s < kBackStages; ++s)
        fetch(blockIdx.x + (int64_t)s * gridDim.x, s);
    int stage = 0, par = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, par ^= 1) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kBackStages - 1) : "memory");
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int g = k * nt + tid;
            if (g < groups) {
                float ga[8], fy[8], fh[8];
                load_gain<8>(a.gain, a.gbf16, g * 8, ga);
                unpack<XT, 8>(held(stage, 0, g), fy);
                unpack<XT, 8>(held(stage, 1, g), fh);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ss = fmaf(fh[e], fh[e], ss);
                    dot = fmaf(fy[e] * ga[e], fh[e], dot);
                }
            }
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
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int g = k * nt + tid;
            if (g < groups) {
                float ga[8], fy[8], fh[8], o[8];
                load_gain<8>(a.gain, a.gbf16, g * 8, ga);
                unpack<XT, 8>(held(stage, 0, g), fy);
                unpack<XT, 8>(held(stage, 1, g), fh);
                if constexpr (RES)
                    unpack<XT, 8>(held(stage, 2, g), o);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = r * fmaf(-fh[e], c, fy[e] * ga[e]);
                    o[e] = RES ? v + o[e] : v;
                    acc[k][e] = fmaf(fy[e], fh[e] * r, acc[k][e]);
                }
                store_group<XT, 8>(static_cast<XT *>(a.dx) + row * a.lddx + g * 8, o);
            }
        }
        fetch(row + (int64_t)kBackStages * gridDim.x, stage);
        stage = stage + 1 == kBackStages ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    float *p = a.partial + (int64_t)blockIdx.x * a.D;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int g = k * nt + tid;
        if (g < groups)
            store_group<float, 8>(p + g * 8, acc[k]);
    }
}

// dgain_j = the sum of the n partial rows of column j: 32 columns a CTA, each
// by 32 threads that take every 32nd row, then joined in order.
__global__ void __launch_bounds__(1024) k_dgain(const float *__restrict__ partial, int n, int D,
                                                float *__restrict__ dgain)
{
    __shared__ float part[32][33];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + c;
    dev::grid_dep_wait();
    float s = 0.f;
    if (col < D)
        for (int k = r; k < n; k += 32)
            s += partial[(int64_t)k * D + col];
    part[r][c] = s;
    __syncthreads();
    // warp r joins column r of the block
    const float t = warp_sum(part[c][r]);
    if (c == 0 && blockIdx.x * 32 + r < D)
        dgain[blockIdx.x * 32 + r] = t;
}

struct BackPlan {
    int vec, nv, tpr, block, grid;
    bool ring;
    size_t smem;
    int64_t parts;  // partial rows
};

// Long rows of whole groups go through the ring: from 1024 columns on (a warp
// of four groups a thread; shorter rows share a CTA), as long as two rows of
// three inputs fit the shared memory.  The rest keeps one row in registers.
BackPlan back_plan(int64_t T, int64_t D, int esize, bool grouped8)
{
    BackPlan p{};
    const size_t smem = (size_t)kBackStages * 3 * D * esize;
    p.ring = grouped8 && D >= 1024 && smem <= 200 << 10;
    p.vec = grouped8 ? 8 : 1;
    p.nv = p.ring ? 4 : grouped8 ? (D <= 2048 ? 1 : D <= 8192 ? 2 : 4) : (D <= 4096 ? 4 : 32);
    p.tpr = threads_per_row(D, p.vec, p.nv);
    p.block = p.ring ? p.tpr : p.tpr < kMinBlock ? kMinBlock : p.tpr;
    const int64_t rpc = p.block / p.tpr;
    const int64_t want = (T + rpc - 1) / rpc;
    int per_sm = p.block >= 1024 ? 1 : 1024 / p.block;
    if (p.ring) {
        p.smem = smem;
        per_sm = (int)((220 << 10) / (smem + 2048));
        const int by_regs = 512 / p.block;
        per_sm = per_sm < by_regs ? per_sm : by_regs;
        per_sm = per_sm > 8 ? 8 : per_sm < 1 ? 1 : per_sm;
    }
    const int64_t most = (int64_t)kSms * per_sm;
    p.grid = (int)(want < most ? want : most);
    p.parts = p.grid * rpc;
    return p;
}

template <typename XT, bool RES>
cudaError_t launch_back(BackArgs a, const BackPlan &p, cudaStream_t stream)
{
    a.tpr = p.tpr;
    auto go = [&](auto kernel) { return launch_k(kernel, dim3(p.grid), dim3(p.block), p.smem, stream, true, a); };
    if (p.ring) {
        auto ring = [&](auto kernel) {
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 << 10);
            return e == cudaSuccess ? go(kernel) : e;
        };
        return p.block <= 256 ? ring(k_rmsnorm_back_ring<XT, RES, 256, 2>) : ring(k_rmsnorm_back_ring<XT, RES, 512, 1>);
    }
    if (p.vec == 8) {
        if (p.nv == 1)
            return go(k_rmsnorm_back<XT, RES, 8, 1, 256>);
        if (p.nv == 2)
            return go(k_rmsnorm_back<XT, RES, 8, 2, 512>);
        return p.block <= 512 ? go(k_rmsnorm_back<XT, RES, 8, 4, 512>) : go(k_rmsnorm_back<XT, RES, 8, 4, 1024>);
    }
    if (p.nv == 4)
        return go(k_rmsnorm_back<XT, RES, 1, 4, 1024>);
    return p.block <= 512 ? go(k_rmsnorm_back<XT, RES, 1, 32, 512>) : go(k_rmsnorm_back<XT, RES, 1, 32, 1024>);
}

// 8-bit rows back as what they stand for: q scale.
template <typename YT, int VEC>
__global__ void __launch_bounds__(256) k_dequantize(const int8_t *__restrict__ q, int64_t ldq,
                                                    const float *__restrict__ scales, int D, YT *__restrict__ y,
                                                    int64_t ldy)
{
    const int64_t row = blockIdx.x;
    const int step = gridDim.y * blockDim.x * VEC;
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    const float s = scales[row];
    for (int col = (blockIdx.y * blockDim.x + threadIdx.x) * VEC; col < D; col += step) {
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
    // four groups a thread in a long call; a few tokens' rows are spread over more CTAs
    const int64_t per = (T <= kSms ? 256 : 1024) * (grouped8 ? 8 : 1);
    const dim3 grid((unsigned)T, (unsigned)((D + per - 1) / per));
    auto go = [&](auto kernel, auto *yt) {
        return launch_k(kernel, grid, dim3(256), 0, (cudaStream_t)stream, true, q, ldq, scales, (int)D, yt, ldy);
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
    for (int k = 0; k < 4; ++k) {
        const int64_t n = back_plan(T, D, k & 1 ? 4 : 2, k >> 1).parts;
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
    const BackPlan p = back_plan(T, D, (int)elem_size(type), grouped8);
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
        e = launch_k(k_dgain, dim3((unsigned)((D + 31) / 32)), dim3(1024), 0, s, true, a.partial, (int)p.parts, (int)D,
                     dgain);
    return launched(e);
}

}  // extern "C"
