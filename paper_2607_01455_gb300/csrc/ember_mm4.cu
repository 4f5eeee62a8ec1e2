// Matrix product with a table in 4 bits:
//
//   out[t][v] = r_v sum_k x[t][k] q_vk s_v,k/group
//
// the logits of a head whose table ember_quantize_rows_nibble has made, for hidden
// states in bf16 or fp32.  On the tensor cores both are fp16 numbers, products
// exact and sums fp32: q s has seven significant bits (ember_quant4.cuh), and the
// hidden states are scaled per token (eight_states).
//
// Three kernels, by the number of tokens and the table's alignment:
//   k_mm4_few  up to 8 columns (a token is a column, or two in fp32): the
//              table is read once and unpacked into the operands of warp-level
//              matrix instructions; bound by HBM.
//   k_mm4_tc   more: tcgen05 on pairs of CTAs; bound by HBM or by the unpacking
//              of the codes up to about 100 tokens, by the tensor cores beyond.
//   k_mm4_any  tables whose rows do not start on 16 bytes.
#include "ember_quant4.cuh"
#include "ember_tc.cuh"

#include <type_traits>

namespace ember {
namespace {

using namespace rows;
using namespace quant4;

constexpr int64_t kMaxMmRows = INT32_MAX - 1024;  // row numbers of a last tile stay within 32 bits
constexpr float kMaxFloat = 0x1.fffffep127f;

struct Mm4Args {
    const void *x;
    const uint8_t *codes, *gscales;
    const float *scales;
    void *out;
    int64_t ldx, ldc, ldg, ldo, T, V;
    int K, log_group, xf32, obf16;
};

__device__ __forceinline__ void store_out(void *out, int obf16, int64_t at, float v)
{
    if (obf16)
        static_cast<unsigned short *>(out)[at] = dev::f2bf(v);
    else
        static_cast<float *>(out)[at] = v;
}

__device__ __forceinline__ float load_x(const void *x, int xf32, int64_t at)
{
    return xf32 ? static_cast<const float *>(x)[at]
                : __uint_as_float((unsigned)static_cast<const unsigned short *>(x)[at] << 16);
}

// Rows at any address: tiles of 64 channels x 16 tokens through shared memory
// as fp32, loaded byte by byte.  Takes what the kernels with 16-byte loads
// cannot.  Sums that pass the floats are formed again with the power of two in the
// rows' scales in the values already (which stay exact), so that large states
// overflow in results alone (in every sum it costs 3 %: 1471 -> 1510 us on 1 x 128256 x 4096).
constexpr int kGV = 64, kGT = 16, kGK = 64;
__device__ __forceinline__ int scale_exponent(float r)  // of a normal number, at most 100
{
    const int e = (int)(__float_as_uint(r) >> 23 & 255u);
    return e == 0 || e == 255 ? 0 : e > 227 ? 100 : e - 127;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

__global__ void __launch_bounds__(256) k_mm4_any(Mm4Args a, unsigned vblocks)
{
    __shared__ float sx[kGT][kGK + 1];
    __shared__ float sw[kGV][kGK + 1];
    __shared__ float sp[kGV];
    const int64_t v0 = (int64_t)(blockIdx.x % vblocks) * kGV, t0 = (int64_t)(blockIdx.x / vblocks) * kGT;
    const int tv = threadIdx.x & 63, tt = threadIdx.x >> 6;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    auto sums = [&](auto scaled) {
        for (int k0 = 0; k0 < a.K; k0 += kGK) {
            for (int i = threadIdx.x; i < kGT * kGK; i += 256) {
                const int r = i / kGK, k = i % kGK;
                sx[r][k] = k0 + k < a.K && t0 + r < a.T ? load_x(a.x, a.xf32, (t0 + r) * a.ldx + k0 + k) : 0.f;
            }
            for (int i = threadIdx.x; i < kGV * kGK / 2; i += 256) {
                const int r = i / (kGK / 2), k = i % (kGK / 2) * 2;
                float lo = 0.f, hi = 0.f;
                if (k0 + k < a.K && v0 + r < a.V) {
                    const unsigned c = a.codes[(v0 + r) * a.ldc + (k0 + k) / 2];
                    float s = e4m3_value(a.gscales[(v0 + r) * a.ldg + ((k0 + k) >> a.log_group)]);
                    if constexpr (decltype(scaled)::value)
                        s *= sp[r];
                    lo = (float)((int)(c & 15u) - 8) * s;
                    hi = k0 + k + 1 < a.K ? (float)((int)(c >> 4) - 8) * s : 0.f;
                }
                sw[r][k] = lo;
                sw[r][k + 1] = hi;
            }
            __syncthreads();
#pragma unroll 8
            for (int k = 0; k < kGK; ++k) {
                const float w = sw[tv][k];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[j] = __fmaf_rn(sx[tt + 4 * j][k], w, acc[j]);
            }
            __syncthreads();
        }
    };
    sums(std::false_type{});
    const int64_t v = v0 + tv;
    float r = v < a.V ? a.scales[v] : 0.f;
    bool past = false;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        past |= !(fabsf(acc[j]) <= kMaxFloat);
    if (__syncthreads_or(past)) {  // or there are infinities or NaN among the inputs
        const int e = scale_exponent(r);
        if (tt == 0)
            sp[tv] = power_of_two(e);
        r *= power_of_two(-e);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc[j] = 0.f;
        __syncthreads();
        sums(std::true_type{});
    }
    if (v >= a.V)
        return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t t = t0 + tt + 4 * j;
        if (t < a.T)
            store_out(a.out, a.obf16, t * a.ldo + v, acc[j] * r);
    }
}

// Hidden states as fp16, scaled by a power of two per token (token_scale) that
// brings the largest into [2^14, 2^15).  A bf16 number is exact then, or below 2^-31 of
// the token's largest and off by 2^-39 of it at most, half of fp16's last step; an fp32
// number becomes a sum of two of 11 bits, p[0] + p[1], off by 2^-23 of itself or by
// as much as a bf16 number, which is more below 2^-16 of the largest.  Eight from k on (zeros behind K),
// in the order 0 4 1 5 2 6 3 7, that of the codes.
template <typename XT> constexpr int kParts = sizeof(XT) == 4 ? 2 : 1;
template <typename XT>
__device__ __forceinline__ void eight_loads(const XT *row, int k, int K, bool wide, float (&f)[8])
{
    if (wide && k + 8 <= K) {
        if constexpr (sizeof(XT) == 2)
            unpack<XT, 8>(load_raw<XT, 8>(row + k), f);
        else {
            const float4 a = *reinterpret_cast<const float4 *>(row + k), b = *reinterpret_cast<const float4 *>(row + k + 4);
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
            f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        }
    } else
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float x[1] = {0.f};
            if (k + e < K)
                unpack<XT, 1>(load_raw<XT, 1>(row + k + e), x);
            f[e] = x[0];
        }
}
template <typename XT>
__device__ __forceinline__ void eight_states(const XT *row, int k, int K, bool wide, float scale,
                                             uint4 (&p)[kParts<XT>])
{
    float f[8];
    eight_loads<XT>(row, k, K, wide, f);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        f[e] *= scale;
#pragma unroll
    for (int q = 0; q < kParts<XT>; ++q) {
        unsigned w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __half2 h = __floats2half2_rn(f[e], f[e + 4]);
            w[e] = *reinterpret_cast<const unsigned *>(&h);
            if (q + 1 < kParts<XT>) {  // what is left
                const float2 g = __half22float2(h);
                f[e] -= g.x;
                f[e + 4] -= g.y;
            }
        }
        p[q] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
// The power of two that brings a token's largest magnitude into [2^14, 2^15)
// (1 for tokens of zeros, of infinities or NaN), and what undoes it.
__device__ __forceinline__ float token_scale(float top)
{
    const int e = (int)(__float_as_uint(top) >> 23);  // of a magnitude or NaN
    if (e == 255 || top == 0.f)
        return 1.f;
    const int k = 127 + 14 + 127 - e;  // tiny ones are brought as far as a float goes
    return __uint_as_float((unsigned)(k > 254 ? 254 : k) << 23);
}

__device__ __forceinline__ uint32_t lds32(const unsigned char *p)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(tc::smem_addr(p)));
    return v;
}
__device__ __forceinline__ uint4 lds128(const unsigned char *p)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(tc::smem_addr(p)));
    return v;
}
// d = a b, or d += a b.  Volatile, as the loads are: in this order the operands
// of the next 32 values are on their way while these are unpacked.
template <bool FIRST>
__device__ __forceinline__ void mma_f16(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0,
                                        unsigned b1)
{
    if constexpr (FIRST)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
            "{%10, %10, %10, %10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                     "{%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// ---------------------------------------------------------------------------
// Few tokens.  A warp multiplies 32 rows of the table by up to 8 columns (a token
// is a column, or two in fp32) with mma.m16n8k16, a box of 32 rows x 256 values at
// a time, which a TMA copy brings to a ring of its own.  The codes become the
// fp16 numbers q (eight_integers); a group's scale multiplies the group's sum,
// in fp32.  (The numbers c 2^-24 that the codes are where they lie would need no
// arithmetic at all, but the tensor cores line subnormals up as if they were
// 2^-14 and lose seven bits of the sum.)
// The order of k within a group is free as long as both operands have the same:
// lane 4 g + t feeds eight values of rows g, g + 8, ... as they are in one word.
// 2^log_ks warps of a CTA share a tile's K and join their sums through shared memory.
// Bound by the instructions that unpack and scale as much as by HBM: 1 x 128256 x 8192
// in groups of 32 100 to 105 us (5.3 to 5.6 TB/s), of 128 88 us (6.1); 8 tokens, whose
// columns' loads from shared memory add up, 139 us.
// A warp whose wait gives up copies and computes nothing more but keeps to the
// barriers, and sets the timeout flag at its end (in the loop the code for it cost
// 5 % and more: 1 x 128256 x 8192 105.6 us with it, 100.2 without).
// ---------------------------------------------------------------------------
constexpr int kFewCols = 8;
constexpr int kFewWarps = 16;
constexpr int kBoxRows = 32, kBoxK = 256, kBoxBytes = kBoxRows * kBoxK / 2;
constexpr int kFewMaxStages = 6;
constexpr size_t kFewSmem = 227 << 10;

struct FewPlan {
    int warps, log_ks, stages;
    int xpitch;              // bytes of a column
    size_t join_at, ring_at;  // in shared memory, behind the columns
    size_t smem;
};

template <typename XT, int LG>
__global__ void __launch_bounds__(kFewWarps * 32, 1)
k_mm4_few(const __grid_constant__ CUtensorMap tm, const Mm4Args a, const FewPlan p, unsigned *flags, uint64_t wait_ns)
{
    constexpr int P = kParts<XT>;
    constexpr int kGroups = kBoxK >> LG;  // of a box
    extern __shared__ unsigned char few_smem_raw[];
    unsigned char *const smem =
        reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(few_smem_raw) + 1023) & ~(uintptr_t)1023);
    float *const join = reinterpret_cast<float *>(smem + p.join_at);  // [warp][row][column]
    __shared__ uint64_t full[kFewWarps][kFewMaxStages];
    __shared__ unsigned tops[kFewCols];  // by token: its largest magnitude, as bits
    __shared__ float back[kFewCols];  // by token: what undoes its scale
    const int T = (int)a.T, cols = T * P;
    const int nthreads = p.warps * 32;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g = lane >> 2,
              t = lane & 3;
    const int kboxes = (a.K + kBoxK - 1) / kBoxK;
    const int ngroups = (a.K + (1 << LG) - 1) >> LG;
    // this warp's boxes of a tile, and its tiles
    const int ks = 1 << p.log_ks, part = warp & (ks - 1);
    const int b0 = part * kboxes >> p.log_ks, b1 = (part + 1) * kboxes >> p.log_ks, nb = b1 - b0;
    const int tiles = (int)((a.V + kBoxRows - 1) / kBoxRows);
    const int per_cta = p.warps >> p.log_ks;
    const int tile0 = blockIdx.x * per_cta + (warp >> p.log_ks), tstep = gridDim.x * per_cta;
    if (lane == 0) {
        for (int s = 0; s < p.stages; ++s)
            tc::mbar_init(tc::smem_addr(&full[warp][s]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < kFewCols)
        tops[threadIdx.x] = 0;
    __syncthreads();
    // the copies: box `pb` of tile `pt` is the next one
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    if (lane == 0)  // the kernel before this one may have written the table, by plain stores
        asm volatile("fence.proxy.async.global;" ::: "memory");
    unsigned char *const ring = smem + p.ring_at + (size_t)warp * p.stages * kBoxBytes;
    const uint32_t ring_addr = tc::smem_addr(ring);
    int pt = tile0, pb = b0, pstage = 0;
    int64_t issued = 0, waited = 0;
    const uint64_t pol = tc::l2_policy(2);
    auto issue = [&]() {
        if (pt >= tiles || nb == 0)
            return;
        if (lane == 0) {
            const uint32_t bar = tc::smem_addr(&full[warp][pstage]);
            tc::mbar_expect_tx(bar, kBoxBytes);
            tc::tma_load_2d_own(ring_addr + pstage * kBoxBytes, &tm, pb * (kBoxK / 2), pt * kBoxRows, bar, pol);
        }
        ++issued;
        pstage = pstage + 1 == p.stages ? 0 : pstage + 1;
        if (++pb == b1) {
            pb = b0;
            pt += tstep;
        }
    };
    for (int s = 0; s < p.stages; ++s)
        issue();

    // the columns: each token's largest magnitude, then the values
    const int units = kboxes * (kBoxK / 8);  // of eight values, whole boxes
    for (int i = threadIdx.x; i < T * units; i += nthreads) {
        const int tok = i / units, k = (i - tok * units) * 8;
        const XT *row = static_cast<const XT *>(a.x) + tok * a.ldx;
        float f[8];
        eight_loads<XT>(row, k, a.K, (uintptr_t)row % 16 == 0, f);
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            m = max_nan(m, fabsf(f[e]));
        // units is a multiple of 32: a warp's are of one token; NaN is the largest of magnitudes' bits
        const unsigned top = __reduce_max_sync(0xffffffffu, __float_as_uint(m) & 0x7FFFFFFFu);
        if (lane == 0)
            atomicMax(&tops[tok], top);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < T * units; i += nthreads) {
        const int tok = i / units, u = i - tok * units;
        const XT *row = static_cast<const XT *>(a.x) + tok * a.ldx;
        const float scale = token_scale(__uint_as_float(tops[tok]));
        if (u == 0)
            back[tok] = 1.f / scale;
        uint4 v[P];
        eight_states<XT>(row, u * 8, a.K, (uintptr_t)row % 16 == 0, scale, v);
#pragma unroll
        for (int q = 0; q < P; ++q)
            *reinterpret_cast<uint4 *>(smem + (size_t)(q * T + tok) * p.xpitch + u * 16) = v[q];
    }
    __syncthreads();

    // 8 bytes of a row's scales a box (4 or 2 for larger groups), by lane and row
    auto scales_of = [&](int tile, int b) {
        uint2 r = make_uint2(0, 0);
        const int64_t v = (int64_t)tile * kBoxRows + lane;
        const int g0 = b * kGroups;
        if (tile >= tiles || v >= a.V)
            return r;
        const uint8_t *q = a.gscales + v * a.ldg + g0;
        if (g0 + kGroups <= ngroups) {
            if constexpr (kGroups == 8)
                r = __ldg(reinterpret_cast<const uint2 *>(q));
            else if constexpr (kGroups == 4)
                r.x = __ldg(reinterpret_cast<const unsigned *>(q));
            else
                r.x = __ldg(reinterpret_cast<const unsigned short *>(q));
        } else
#pragma unroll
            for (int e = 0; e < kGroups; ++e)
                if (g0 + e < ngroups)
                    (e < 4 ? r.x : r.y) |= (unsigned)q[e] << (8 * (e & 3));
        return r;
    };
    const unsigned char *const xcol = smem + (size_t)(g < cols ? g : 0) * p.xpitch + t * 16;
    auto tile_sync = [&]() {  // the warps that share a tile: at most 8 such sets
        if (ks == 1)
            __syncwarp();
        else
            asm volatile("bar.sync %0, %1;" ::"r"(1 + (warp >> p.log_ks)), "r"(ks * 32) : "memory");
    };
    // any wait counts as longer than a limit below a microsecond, whether or not a copy
    // is there at the first look
    bool failed = wait_ns < 1000;
    int stage = 0;
    uint32_t phase = 0;
    uint2 snext = nb > 0 ? scales_of(tile0, b0) : make_uint2(0, 0);
    for (int tile = tile0; (tile - tile0) + blockIdx.x * per_cta < tiles; tile += tstep) {  // the same rounds for all warps
        float acc[2][4];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            acc[e >> 2][e & 3] = 0.f;
        if (tile < tiles)
            for (int b = b0; b < b1; ++b) {
                const uint2 sc = snext;
                snext = b + 1 < b1 ? scales_of(tile, b + 1) : scales_of(tile + tstep, b0);
                if (!failed) {
                    failed = !tc::mbar_spin_alone(tc::smem_addr(&full[warp][stage]), phase, wait_ns);
                    failed = __any_sync(0xffffffffu, failed);
                }
                if (failed)
                    break;
                ++waited;
                float sg[kGroups];  // of this lane's row
#pragma unroll
                for (int e = 0; e < kGroups; e += 2) {
                    const float2 two = e4m3_pair(e < 4 ? sc.x : sc.y, e & 3);
                    sg[e] = two.x;
                    sg[e + 1] = two.y;
                }
                const unsigned char *box = ring + stage * kBoxBytes + g * 128 + t * 4;
                const unsigned char *xb = xcol + (size_t)b * (kBoxK * 2);
                uint32_t wnext[4];
                uint4 xnext;
                auto ahead = [&](int j) {
                    const unsigned char *at = box + ((j ^ g) << 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        wnext[e] = lds32(at + e * 1024);
                    xnext = lds128(xb + j * 64);
                };
                ahead(0);
#pragma unroll
                for (int gr = 0; gr < kGroups; ++gr) {
                    float d[2][4];
#pragma unroll
                    for (int h = 0; h < (1 << LG) / 32; ++h) {  // 32 values: a word a lane and row
                        const int j = gr * ((1 << LG) / 32) + h;
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = wnext[e];
                        const uint4 x = xnext;
                        if (j + 1 < kBoxK / 32)
                            ahead(j + 1);
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            uint32_t u[4], v[4];
                            eight_integers(w[2 * m], u);
                            eight_integers(w[2 * m + 1], v);
                            if (h == 0)
                                mma_f16<true>(d[m], u[0], v[0], u[1], v[1], x.x, x.y);
                            else
                                mma_f16<false>(d[m], u[0], v[0], u[1], v[1], x.x, x.y);
                            mma_f16<false>(d[m], u[2], v[2], u[3], v[3], x.z, x.w);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {  // rows g + 8 e
                        const float f = __shfl_sync(0xffffffffu, sg[gr], g + 8 * e);
                        float(&o)[4] = acc[e >> 1];
                        const float(&i)[4] = d[e >> 1];
                        o[(e & 1) * 2] = __fmaf_rn(i[(e & 1) * 2], f, o[(e & 1) * 2]);
                        o[(e & 1) * 2 + 1] = __fmaf_rn(i[(e & 1) * 2 + 1], f, o[(e & 1) * 2 + 1]);
                    }
                }
                __syncwarp();  // the box has been read
                issue();
                if (++stage == p.stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        float *mine = join + warp * (kBoxRows * kFewCols);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            *reinterpret_cast<float2 *>(mine + (g + 8 * e) * kFewCols + 2 * t) =
                make_float2(acc[e >> 1][(e & 1) * 2], acc[e >> 1][(e & 1) * 2 + 1]);
        tile_sync();
        // a thread per row and token: parts of K in order, each with the parts of
        // an fp32 number
        const float *tile_join = join + (warp & ~(ks - 1)) * (kBoxRows * kFewCols);
        for (int o = part * 32 + lane; o < kBoxRows * T; o += ks * 32) {
            const int r = o % kBoxRows, tok = o / kBoxRows;
            float sum = 0.f;
            for (int k = 0; k < ks; ++k)
#pragma unroll
                for (int q = 0; q < P; ++q)
                    sum += tile_join[(k * kBoxRows + r) * kFewCols + q * T + tok];
            const int64_t v = (int64_t)tile * kBoxRows + r;
            if (v < a.V)
                store_out(a.out, a.obf16, tok * a.ldo + v, sum * a.scales[v] * back[tok]);
        }
        tile_sync();
    }
    if (failed && issued > 0 && lane == 0)
        atomicOr(flags, kFlagTimeout);
    // copies that a warp which gave up has not waited for
    if (lane == 0)
        for (int64_t i = waited; i < issued; ++i)
            tc::mbar_wait_final(tc::smem_addr(&full[warp][i % p.stages]), (uint32_t)(i / p.stages & 1));
}

// ---------------------------------------------------------------------------
// Many tokens, on the tensor cores.  A pair of CTAs multiplies 256 rows of the
// table (the M of tcgen05.mma.cta_group::2, 128 rows in each CTA) by N tokens.
// Per block of 256 along K each CTA
//   - gets its 128 rows of codes, 16 KiB, by TMA into 128-byte swizzled shared
//     memory;
//   - widens them to q s / 8 in fp16 in registers (a thread per row and quarter, 64
//     values) and stores them in tensor memory as the A operand, in slots of 128
//     columns;
//   - gets its half of the tokens' block by TMA, already fp16 in the order of
//     the codes (k_split4 writes them once per call), one block after another
//     for the two parts of fp32 numbers, both multiplied with the same A.
// A block costs the warp that issues the MMAs about 1000 clocks in waits, commits
// and the loop, whatever N: hence blocks of 256 and not of 128.
// The group scales, 32 of each row at a time, come by TMA too.  (Loaded by the
// widening threads themselves, 16 bytes a row, they were fetched several times
// over: 64 x 128256 x 4096 125 us.)
// Roles (768 threads per CTA, one CTA per SM, persistent over tiles):
//   warps 0, 2, 3  issue the TMA loads of the codes, the tokens and the scales:
//                three rings
//   warp 1       allocates tensor memory; in the even CTA issues the MMAs
//   warps 4-7    epilogue: scales and stores an accumulator (two of them, so
//                that it overlaps the next tile's MMAs)
//   warps 8-23   widen: eight warps the even blocks, eight the odd ones, four of
//                them each half; most of a warp's time for a block are waits and
//                barriers (1100 clocks of 1770 with all sixteen at every block)
// Measured: 64 x 128256 x 4096 81 us (830 TFLOP/s, 3.6 TB/s; tensor pipes busy 38 %
// of the time, HBM 44 %, ALU 60 %: the widening warps' chain of wait, unpack, store and an
// arrival at both CTAs bounds it), 256 x 32000 x 4096 62 us (1090), 2048 x 32000 x 4096 327 to
// 360 us by the power limit (1490 to 1640; 0.77 to 0.85 of the measured peak); fp32 states
// and outputs 600 x 32000 x 4096 198 us (1590 with both parts).
// Every wait is bounded; one that gives up sets the timeout flag, stops every
// role, and the kernel returns after its copies and MMAs in flight are done.
// The two CTAs may then have issued different numbers of copies of the tokens,
// whose bytes complete on one barrier: the even CTA evens the counts out.
// ---------------------------------------------------------------------------
using namespace tc;

constexpr int kTcRows = 128;  // rows of the table per CTA
constexpr int kTcK = 256;     // block along K
constexpr int kTcThreads = 768;
constexpr int kTcMaxN = 128;  // tokens of a tile: two accumulators and two slots of A fill tensor memory
constexpr int kTcMaxStages = 12, kTcMaxSlots = 3;
constexpr int kTcWBytes = kTcRows * kTcK / 2;  // a block of codes
constexpr int kTcSBox = 32;  // scales of a row in a stage of the scales
constexpr int kTcSBytes = kTcRows * kTcSBox, kSRing = 3;
constexpr int kTcSlotCols = kTcK / 2;      // a block of A as fp16 pairs
constexpr size_t kTcSmem = 227 << 10;

struct Tc4Tail {
    uint64_t wfull[kTcMaxStages];   // each CTA: its rows of the table landed
    uint64_t wempty[kTcMaxStages];  // each CTA: read by the eight warps that widen it
    uint64_t sfull[kSRing], sempty[kSRing];  // each CTA: the scales, as the codes
    uint64_t bfull[kTcMaxStages];   // even CTA: both halves of the tokens landed
    uint64_t bempty[kTcMaxStages];  // each CTA: the MMAs of the stage are done
    uint64_t afull[kTcMaxSlots];    // even CTA: both CTAs' A slots written
    uint64_t aempty[kTcMaxSlots];   // each CTA: the MMAs of the slot are done
    uint64_t tfull[2], tempty[2];   // accumulators
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
    int64_t issued[2];   // in the even CTA: blocks of the tokens whose copies each CTA has issued
    int64_t gave_up[2];  // in both: whether a wait of either CTA gave up
    float back[4][kTcMaxN];  // the tokens' factors of a tile, a copy per epilogue warp
};

struct Tc4Args {
    const float *scales, *back;  // by row of the table; by token: what undoes its scale
    void *out;
    unsigned *flags;
    int64_t ldo;
    int T, V, K;
    int N, ntb, wstages, bstages, slots, obf16;
    int parts;    // of a hidden state: 1 or 2
    int split;    // parts of K; with more than one, each writes its sums to
    float *part;  // part[split][T][V]
    uint32_t idesc;
    uint64_t wait_ns;
};

// The tokens as fp16, [part][T] rows of kp (a multiple of 8) values in the
// codes' order, zeros behind K, and what undoes their scales and the table's
// eighth.  A CTA per token.
template <typename XT>
__global__ void __launch_bounds__(256) k_split4(const XT *__restrict__ x, int64_t ldx, int64_t T, int K, int kp,
                                                uint4 *__restrict__ xh, float *__restrict__ back)
{
    __shared__ float tops[8];
    const int64_t t = blockIdx.x;
    const XT *row = x + t * ldx;
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    const bool wide = (uintptr_t)row % 16 == 0;
    float m = 0.f;
    for (int k = threadIdx.x * 8; k < K; k += 256 * 8) {
        float f[8];
        eight_loads<XT>(row, k, K, wide, f);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            m = max_nan(m, fabsf(f[e]));
    }
    m = warp_max_nan(m);
    if ((threadIdx.x & 31) == 0)
        tops[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w)
        m = max_nan(m, tops[w]);
    const float scale = token_scale(m);
    if (threadIdx.x == 0)
        back[t] = 8.f / scale;
    for (int k = threadIdx.x * 8; k < kp; k += 256 * 8) {
        uint4 p[kParts<XT>];
        eight_states<XT>(row, k, K, wide, scale, p);
#pragma unroll
        for (int q = 0; q < kParts<XT>; ++q)
            xh[((q * T + t) * kp + k) / 8] = p[q];
    }
}

__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(unsigned short *p, float v) { *p = dev::f2bf(v); }
// 32 tokens of one channel's column, scaled, into nt rows of the output.  The
// lanes of a warp hold 32 neighbouring channels: a store per token writes 64 or
// 128 bytes of a row in one piece.
template <typename T>
__device__ __forceinline__ void write_cols4(T *p, int64_t ldo, float (&d)[32], const float *back, float r, int nt, bool on)
{
    const f2 r2 = make2(r, r);
#pragma unroll
    for (int e = 0; e < 32; e += 4) {  // the power of two last: one rounding, and large states overflow in results alone
        const float4 b = *reinterpret_cast<const float4 *>(back + e);
        split2(mul2(mul2(make2(d[e], d[e + 1]), r2), make2(b.x, b.y)), d[e], d[e + 1]);
        split2(mul2(mul2(make2(d[e + 2], d[e + 3]), r2), make2(b.z, b.w)), d[e + 2], d[e + 3]);
    }
    if (!on)
        return;
    if (nt >= 32) {
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            put(p, d[e]);
            p += ldo;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 32; ++e)
            if (e < nt) {
                put(p, d[e]);
                p += ldo;
            }
    }
}

// Registers of the warps where the epilogue keeps sums: what the block is
// launched with, 80 a thread, shared out again.
constexpr int kTcRegs = 80, kTcRegsFew = 56, kTcRegsWiden = 64, kTcRegsSums = 168;
static_assert(128 * kTcRegsFew + 128 * kTcRegsSums + 512 * kTcRegsWiden <= kTcThreads * kTcRegs, "a raise waits for registers given up");
// Not in builds without optimisation, whose code for the roles fits no share.
#ifdef EMBER_OPTIMIZED
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
#else
template <int N>
__device__ __forceinline__ void regs_down() {}
template <int N>
__device__ __forceinline__ void regs_up() {}
#endif

// SPLIT: the calls whose K is in parts; the others divide by nothing per tile.
// SUMS: outputs in fp32.  The tensor cores cut a sum off after each step of 16
// products; over a whole K that costs more than fp32 sums do (33 x 10007 x 2049:
// 4e-6 of the result against 8e-7), so an accumulator holds one block of 256
// and the epilogue adds the blocks up in registers, rounded.
template <bool SPLIT, int LG, bool SUMS>
__global__ void __launch_bounds__(kTcThreads, 1)
k_mm4_tc(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_s,
         const __grid_constant__ CUtensorMap tm_x, const Tc4Args a)
{
    extern __shared__ unsigned char tc_smem_raw[];
    unsigned char *smem =
        reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(tc_smem_raw) + 1023) & ~(uintptr_t)1023);
    const int b_box = a.N / 2 * 128;  // N / 2 tokens x 64 fp16; four to a block
    unsigned char *bring = smem + (size_t)a.wstages * kTcWBytes;
    unsigned char *sring = bring + (size_t)a.bstages * 4 * b_box;
    Tc4Tail *tail = reinterpret_cast<Tc4Tail *>(sring + kSRing * kTcSBytes);
    constexpr int kSPer = kTcK >> LG;             // scales of a block: 8, 4 or 2
    constexpr int kSBlocks = kTcSBox / kSPer;     // blocks that a stage of the scales lasts for
    volatile int *abort = &tail->abort;

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);  // uniform, and seen to be
    const int lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank();
    const bool leader = rank == 0;
    const int split = SPLIT ? a.split : 1;
    const int ntiles = (a.V + 2 * kTcRows - 1) / (2 * kTcRows) * a.ntb * split;  // tiles times parts of K
    const int kblocks = (a.K + kTcK - 1) / kTcK;
    auto first_block = [&](int tile) { return (int)((int64_t)(tile % split) * kblocks / split); };
    auto end_block = [&](int tile) { return (int)((int64_t)(tile % split + 1) * kblocks / split); };
    const int tile0 = (int)cluster_id(), tstep = (int)cluster_count();

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.wstages; ++s) {
            mbar_init(smem_addr(&tail->wfull[s]), 1);
            mbar_init(smem_addr(&tail->wempty[s]), 8);
        }
        for (int s = 0; s < kSRing; ++s) {
            mbar_init(smem_addr(&tail->sfull[s]), 1);
            mbar_init(smem_addr(&tail->sempty[s]), 16);
        }
        for (int s = 0; s < a.bstages; ++s) {
            mbar_init(smem_addr(&tail->bfull[s]), 1);
            mbar_init(smem_addr(&tail->bempty[s]), 1);
        }
        for (int s = 0; s < a.slots; ++s) {
            mbar_init(smem_addr(&tail->afull[s]), 16);  // eight warps in each CTA
            mbar_init(smem_addr(&tail->aempty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_addr(&tail->tfull[s]), 1);
            mbar_init(smem_addr(&tail->tempty[s]), 8);
        }
        mbar_init(smem_addr(&tail->drain), 1);
        tail->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_w)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_s)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_x)) : "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         smem_addr(&tail->tmem_base)),
                     "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // no peer may signal this CTA's barriers before they are initialised
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tail->tmem_base, 0);
    const uint32_t slot0 = tmem + 2 * a.N;
    dev::grid_dep_wait();
    dev::grid_dep_launch();

    if (warp < 4) {
    if constexpr (SUMS)
        regs_down<kTcRegsFew>();
    if (warp == 3 && lane == 0) {
        // ---------------- TMA producer of the scales (both CTAs) ----------------
        int stage = 0;
        uint32_t phase = 0;
        int64_t issued = 0;
        asm volatile("fence.proxy.async.global;" ::: "memory");  // as below
        const uint64_t pol = l2_policy(a.ntb > 1 ? 0 : 2);
        bool ok = true;
        for (int tile = tile0; tile < ntiles && ok; tile += tstep) {
            const int vrow = (tile / split / a.ntb * 2 + rank) * kTcRows;
            for (int c = first_block(tile) / kSBlocks; c <= (end_block(tile) - 1) / kSBlocks; ++c) {
                if (!mbar_spin(smem_addr(&tail->sempty[stage]), phase ^ 1u, abort, a.wait_ns)) {
                    ok = false;
                    break;
                }
                const uint32_t bar = smem_addr(&tail->sfull[stage]);
                ++issued;
                mbar_expect_tx(bar, kTcSBytes);
                tma_load_2d(smem_addr(sring + (size_t)stage * kTcSBytes), &tm_s, c * kTcSBox, vrow, bar, pol);
                if (++stage == kSRing) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
        if (!ok)
            set_timeout(abort, a.flags);
        for (int64_t i = issued > kSRing ? issued - kSRing : 0; i < issued; ++i)
            mbar_wait_final(smem_addr(&tail->sfull[i % kSRing]), (uint32_t)(i / kSRing & 1));
    } else if ((warp == 0 || warp == 2) && lane == 0) {
        // ---------------- TMA producers (both CTAs) ----------------
        const bool tokens = warp == 2;
        const int stages = tokens ? a.bstages : a.wstages;
        uint64_t *full = tokens ? tail->bfull : tail->wfull, *empty = tokens ? tail->bempty : tail->wempty;
        int stage = 0;
        uint32_t phase = 0;
        int64_t issued = 0;  // blocks whose copies were issued
        // the tokens were written by plain stores, and the table may have been
        asm volatile("fence.proxy.async.global;" ::: "memory");
        // the table streams when every block is read once
        const uint64_t pol = l2_policy(tokens ? 1 : a.ntb > 1 ? 0 : 2);
        bool ok = true;
        for (int tile = tile0; tile < ntiles && ok; tile += tstep) {
            const int vrow = (tile / split / a.ntb * 2 + rank) * kTcRows;
            const int trow = tile / split % a.ntb * a.N + rank * (a.N / 2);
            const int parts = tokens ? a.parts : 1, n1 = end_block(tile) * parts;
            for (int n = first_block(tile) * parts; n < n1; ++n) {
                if (!mbar_spin(smem_addr(&empty[stage]), phase ^ 1u, abort, a.wait_ns)) {
                    ok = false;
                    break;
                }
                const uint32_t bar = smem_addr(&full[stage]);
                ++issued;
                if (tokens) {
                    if (leader)
                        mbar_expect_tx(bar, 8 * b_box);  // both CTAs' halves, four boxes each
                    const uint32_t dst = smem_addr(bring + (size_t)stage * 4 * b_box);
                    const uint32_t lead = mapa_rank(bar, 0);
                    // the second part of fp32 numbers first: what the sum loses depends
                    // on its size at each step
                    const int kb = parts == 1 ? n : n / 2, row = parts == 1 ? trow : (~n & 1) * a.T + trow;
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        tma_load_2d(dst + q * b_box, &tm_x, kb * kTcK + q * 64, row, lead, pol);
                } else {
                    mbar_expect_tx(bar, kTcWBytes);
                    tma_load_2d(smem_addr(smem + (size_t)stage * kTcWBytes), &tm_w, n * (kTcK / 2), vrow, bar, pol);
                }
                if (++stage == stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
        if (!ok)
            set_timeout(abort, a.flags);
        if (tokens)
            store_remote_i64(&tail->issued[rank], 0, issued);
        else  // this CTA's copies of the table land before it goes on
            for (int64_t i = issued > stages ? issued - stages : 0; i < issued; ++i)
                mbar_wait_final(smem_addr(&full[i % stages]), (uint32_t)(i / stages & 1));
    } else if (warp == 1 && leader) {
        // ---------------- MMA issuer (even CTA) ----------------
        // The whole warp runs the loop and one lane issues, so that operands
        // that are the same in every lane stay in uniform registers.
        int stage = 0, slot = 0, acc = 0;
        uint32_t phase = 0, aphase = 0, acc_phase = 0;
        bool ok = true;
        const uint32_t bring_addr = smem_addr(bring);
        const uint32_t full0 = smem_addr(&tail->bfull[0]), afull0 = smem_addr(&tail->afull[0]);
        for (int tile = tile0; tile < ntiles && ok; tile += tstep) {
            uint32_t d_tmem = 0;
            auto take = [&]() {  // the next accumulator
                ok = mbar_spin(smem_addr(&tail->tempty[acc]), acc_phase ^ 1u, abort, a.wait_ns);
                ok = __all_sync(0xffffffffu, ok);
                d_tmem = tmem + (uint32_t)(acc * a.N);
            };
            auto give = [&]() {
                if (elect_one())
                    mma_commit_mc(smem_addr(&tail->tfull[acc]));
                __syncwarp();
                if (++acc == 2) {
                    acc = 0;
                    acc_phase ^= 1u;
                }
            };
            if constexpr (!SUMS)
                take();
            const int kb0 = first_block(tile), kb1 = end_block(tile);
            for (int kb = kb0; kb < kb1 && ok; ++kb) {
                if constexpr (SUMS) {
                    take();
                    if (!ok)
                        break;
                }
                ok = mbar_spin(afull0 + slot * 8, aphase, abort, a.wait_ns);
                const uint32_t a_base = slot0 + (uint32_t)(slot * kTcSlotCols);
                for (int p = 0; p < a.parts; ++p) {
                    ok = ok && mbar_spin(full0 + stage * 8, phase, abort, a.wait_ns);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok)
                        break;
                    tc_fence_after();
                    const uint64_t b_desc = k_major_sw128_desc(bring_addr + stage * 4 * b_box);
                    if (elect_one()) {
                        auto step = [&](int k) {
                            mma_f16_ta(d_tmem, a_base + k * 8, b_desc + (uint64_t)((k >> 2) * (b_box >> 4) + 2 * (k & 3)),
                                       a.idesc, ((SUMS ? 0 : kb - kb0) | p | k) != 0);
                        };
                        const int steps = (a.K - kb * kTcK + 15) / 16;  // what the last block has of K
                        if (steps >= kTcK / 16)
#pragma unroll
                            for (int k = 0; k < kTcK / 16; ++k)
                                step(k);
                        else
                            for (int k = 0; k < steps; ++k)
                                step(k);
                        mma_commit_mc(smem_addr(&tail->bempty[stage]));
                        if (p == a.parts - 1)
                            mma_commit_mc(smem_addr(&tail->aempty[slot]));
                    }
                    __syncwarp();
                    if (++stage == a.bstages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (++slot == a.slots) {
                    slot = 0;
                    aphase ^= 1u;
                }
                if (SUMS && ok)
                    give();
            }
            if (!ok)
                break;
            if constexpr (!SUMS)
                give();
        }
        if (elect_one()) {
            if (!ok)
                set_timeout(abort, a.flags);
            mma_commit(smem_addr(&tail->drain));
            mbar_wait_final(smem_addr(&tail->drain), 0);
        }
        __syncwarp();
    }
    } else if (warp >= 8) {
        // ---------------- widening: codes into tensor memory ----------------
        if constexpr (SUMS)
            regs_down<kTcRegsWiden>();
        const int q = warp & 3;
        const int half = (warp - 8) >> 2 & 1;  // of a block: two quarters, one after the other
        const bool odd = warp >= 16;           // which of the blocks
        const int r = q * 32 + lane;
        const uint32_t lanes = (uint32_t)(q * 32) << 16;
        int stage = 0, slot = 0, sstage = 0;
        uint32_t phase = 0, aphase = 0, sphase = 0;
        bool ok = true, mine = !odd;
        const unsigned char *srow = sring + r * kTcSBox;
        for (int tile = tile0; tile < ntiles && ok; tile += tstep) {
            const int kb0 = first_block(tile), kb1 = end_block(tile);
            for (int kb = kb0; kb < kb1; ++kb, mine = !mine) {
                // a stage of the scales is waited for and given back by all, so that
                // nobody gives one back twice before the others have once
                if (kb == kb0 || kb % kSBlocks == 0) {
                    ok = mbar_spin(smem_addr(&tail->sfull[sstage]), sphase, abort, a.wait_ns);
                    // the lanes give up together: here, or with the vote on a block of their own
                    // (as a vote: 64 x 128256 x 4096 80.4 us, as a sum 79.5)
                    if (!mine)
                        ok = !__reduce_or_sync(0xffffffffu, !ok);
                }
                if (mine) {
                    ok = ok && mbar_spin(smem_addr(&tail->wfull[stage]), phase, abort, a.wait_ns);
                    const unsigned char *row = smem + (size_t)stage * kTcWBytes + r * 128;
                    const unsigned char *sblock = srow + sstage * kTcSBytes + kb * kSPer % kTcSBox;
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const int quarter = half * 2 + p;
                        uint4 raw[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            raw[c] = *reinterpret_cast<const uint4 *>(row + (((quarter * 2 + c) ^ (r & 7)) << 4));
                        // the scales of these 64 values: two bytes, or one of a pair's
                        const int at = LG == 5 ? quarter * 2 : LG == 6 ? quarter : half;
                        const uint32_t two = *reinterpret_cast<const uint16_t *>(sblock + (at & ~1));
                        const Scale4 s0 = scale4(two, LG == 5 ? 0 : at & 1);
                        const Scale4 s1 = LG == 5 ? scale4(two, 1) : s0;
                        uint32_t w[32];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const unsigned x[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                unsigned o[4];
                                eight_values(x[e], c ? s1 : s0, o);
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    w[c * 16 + e * 4 + j] = o[j];
                            }
                        }
                        if (p == 0) {
                            ok = ok && mbar_spin(smem_addr(&tail->aempty[slot]), aphase ^ 1u, abort, a.wait_ns);
                            ok = __all_sync(0xffffffffu, ok);
                            if (!ok)
                                break;
                            tc_fence_after();
                        }
                        tmem_store32(slot0 + (uint32_t)(slot * kTcSlotCols + quarter * 32) + lanes, w);
                    }
                    if (!ok)
                        break;
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive_remote(mapa_rank(smem_addr(&tail->afull[slot]), 0));
                        mbar_arrive(smem_addr(&tail->wempty[stage]));
                    }
                }
                if (kb + 1 == kb1 || (kb + 1) % kSBlocks == 0) {
                    __syncwarp();
                    if (lane == 0)
                        mbar_arrive(smem_addr(&tail->sempty[sstage]));
                    if (++sstage == kSRing) {
                        sstage = 0;
                        sphase ^= 1u;
                    }
                }
                if (++stage == a.wstages) {
                    stage = 0;
                    phase ^= 1u;
                }
                if (++slot == a.slots) {
                    slot = 0;
                    aphase ^= 1u;
                }
            }
        }
        if (!ok && lane == 0 && !*abort)
            set_timeout(abort, a.flags);
    } else {
        // ---------------- epilogue (both CTAs) ----------------
        if constexpr (SUMS)
            regs_up<kTcRegsSums>();
        const int q = warp - 4;
        int acc = 0;
        uint32_t acc_phase = 0;
        bool ok = true;
        // waits for an accumulator; gives it back
        auto take = [&]() {
            ok = mbar_spin(smem_addr(&tail->tfull[acc]), acc_phase, abort, a.wait_ns);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok && lane == 0 && !*abort)
                set_timeout(abort, a.flags);
            tc_fence_after();
            return tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * a.N);
        };
        auto give = [&]() {
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                mbar_arrive_remote(mapa_rank(smem_addr(&tail->tempty[acc]), 0));
            if (++acc == 2) {
                acc = 0;
                acc_phase ^= 1u;
            }
        };
        for (int tile = tile0; tile < ntiles && ok; tile += tstep) {
            const int v = (tile / split / a.ntb * 2 + rank) * kTcRows + q * 32 + lane;
            const int t0 = tile / split % a.ntb * a.N;
            const bool whole = split == 1;
            const float rv = !whole ? 1.f : v < a.V ? a.scales[v] : 0.f;
            const int nt = a.T - t0 < a.N ? a.T - t0 : a.N;  // tokens of this tile
            float *back = tail->back[q];
            __syncwarp();  // the last tile's have been read
            for (int k = lane; k < a.N; k += 32)
                back[k] = !whole ? 1.f : k < nt ? a.back[t0 + k] : 0.f;
            __syncwarp();
            const int64_t at = (int64_t)t0 * a.ldo + v;
            float *part = a.part + ((int64_t)(tile % split) * a.T + t0) * a.V + v;
            if constexpr (SUMS) {
                float sum[kTcMaxN / 32][32];
#pragma unroll
                for (int c = 0; c < kTcMaxN / 32; ++c)
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        sum[c][e] = 0.f;
                for (int kb = first_block(tile), kb1 = end_block(tile); kb < kb1; ++kb) {
                    const uint32_t d_tmem = take();
                    if (!ok)
                        break;
#pragma unroll
                    for (int c = 0; c < kTcMaxN / 32; ++c)
                        if (c * 32 < a.N) {
                            float d[32];
                            tmem_load32(d_tmem + c * 32, d);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                sum[c][e] += d[e];
                        }
                    give();
                }
                if (!ok)
                    break;
#pragma unroll
                for (int c = 0; c < kTcMaxN / 32; ++c)
                    if (c * 32 < nt)
                        write_cols4(whole ? static_cast<float *>(a.out) + at + c * 32 * a.ldo : part + (int64_t)c * 32 * a.V,
                                    whole ? a.ldo : (int64_t)a.V, sum[c], back + c * 32, rv, nt - c * 32, v < a.V);
            } else {
                const uint32_t d_tmem = take();
                if (!ok)
                    break;
                for (int c = 0; c < nt; c += 32) {
                    float d[32];
                    tmem_load32(d_tmem + c, d);
                    if (whole)
                        write_cols4(static_cast<unsigned short *>(a.out) + at + c * a.ldo, a.ldo, d, back + c, rv, nt - c, v < a.V);
                    else
                        write_cols4(part + (int64_t)c * a.V, (int64_t)a.V, d, back + c, rv, nt - c, v < a.V);
                }
                give();
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (threadIdx.x < 2)
        store_remote_i64(&tail->gave_up[rank], threadIdx.x, *abort);
    cluster_sync();  // the pair's MMAs and arrivals are over on both sides
    if (tail->gave_up[0] | tail->gave_up[1]) {
        // the last copies of the tokens, of both CTAs; a block that only one of
        // them has issued lacks the other's bytes (or the arrival itself)
        if (leader && threadIdx.x == 0) {
            const int64_t n0 = tail->issued[0], n1 = tail->issued[1], n = n0 > n1 ? n0 : n1;
            for (int64_t i = n > a.bstages ? n - a.bstages : 0; i < n; ++i) {
                const uint32_t bar = smem_addr(&tail->bfull[i % a.bstages]);
                if (i >= n0)
                    mbar_expect_tx(bar, 4 * b_box);  // a CTA's half of a block
                else if (i >= n1)
                    mbar_complete_tx(bar, 4 * b_box);
                mbar_wait_final(bar, (uint32_t)(i / a.bstages & 1));
            }
        }
        __syncthreads();
        cluster_sync();
    }
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// The parts of K joined, in order, and scaled.
__global__ void __launch_bounds__(256) k_mm4_join(const Tc4Args a)
{
    const int v = blockIdx.x * 256 + threadIdx.x;
    const int64_t t = blockIdx.y;
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    if (v >= a.V)
        return;
    float s = 0.f;
#pragma unroll 4
    for (int k = 0; k < a.split; ++k)
        s += a.part[((int64_t)k * a.T + t) * a.V + v];
    store_out(a.out, a.obf16, t * a.ldo + v, s * a.scales[v] * a.back[t]);
}

// Blocks of tokens, all of one width N (a multiple of 32).  One when they fit;
// otherwise the widths are weighed by the rounds that the SM pairs need for the
// tiles and by what a round costs, its N and about 24 tokens' worth of fixed
// work, as for the 8-bit product.
void token_blocks4(int64_t T, int64_t vblocks, int *ntb, int *N)
{
    int64_t best = INT64_MAX;
    for (int n = kTcMaxN; n >= 64; n -= 32) {
        const int64_t blocks = (T + n - 1) / n;
        const int width = (int)(((T + blocks - 1) / blocks + 31) / 32 * 32);
        const int64_t rounds = (vblocks * blocks + kSms / 2 - 1) / (kSms / 2);
        if (rounds * (width + 24) < best) {
            best = rounds * (width + 24);
            *ntb = (int)blocks;
            *N = width;
        }
    }
}

int64_t split_cols(int64_t K) { return (K + 7) / 8 * 8; }

// Plan of a call on the tensor cores.  Where the tiles leave half of the SM
// pairs or more without one, K is split among them, 4 blocks or more to a
// part, if that takes 6 blocks or more off every pair (about what the joining
// launch costs).
struct Tc4Plan {
    int ntb, N, split;
    size_t back_at, part_at, bytes;  // where the factors and the parts begin in the workspace, and its size
};
Tc4Plan tc4_plan(int64_t T, int64_t V, int64_t K, bool xf32)
{
    Tc4Plan p;
    const int64_t vblocks = (V + 2 * kTcRows - 1) / (2 * kTcRows), kblocks = (K + kTcK - 1) / kTcK;
    token_blocks4(T, vblocks, &p.ntb, &p.N);
    const int64_t tiles = vblocks * p.ntb;
    const int64_t by_pairs = kSms / 2 / tiles, by_blocks = kblocks / 4;
    p.split = (int)(by_pairs < by_blocks ? by_pairs : by_blocks);
    if (p.split < 2 || kblocks - (kblocks + p.split - 1) / p.split < 6)
        p.split = 1;
    p.back_at = ((size_t)(T * split_cols(K)) * 2 * (xf32 ? 2 : 1) + 255) / 256 * 256;
    p.part_at = p.back_at + ((size_t)T * sizeof(float) + 255) / 256 * 256;
    p.bytes = p.part_at + (p.split > 1 ? (size_t)p.split * T * V * sizeof(float) : 0);
    return p;
}

cudaError_t launch_tc4(const Mm4Args &m, void *workspace, unsigned *flags, cudaStream_t stream)
{
    const int kp = (int)split_cols(m.K), parts = m.xf32 ? 2 : 1;
    const Tc4Plan p = tc4_plan(m.T, m.V, m.K, m.xf32);
    float *back = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + p.back_at);
    cudaError_t e =
        m.xf32 ? launch_k(k_split4<float>, dim3((unsigned)m.T), dim3(256), 0, stream, true,
                          static_cast<const float *>(m.x), m.ldx, m.T, m.K, kp, static_cast<uint4 *>(workspace), back)
               : launch_k(k_split4<bf16_t>, dim3((unsigned)m.T), dim3(256), 0, stream, true,
                          static_cast<const bf16_t *>(m.x), m.ldx, m.T, m.K, kp, static_cast<uint4 *>(workspace), back);
    if (e != cudaSuccess)
        return e;
    Tc4Args a{};
    a.scales = m.scales;
    a.back = back;
    a.out = m.out;
    a.flags = flags;
    a.ldo = m.ldo;
    a.T = (int)m.T;
    a.V = (int)m.V;
    a.K = m.K;
    a.obf16 = m.obf16;
    a.parts = parts;
    a.wait_ns = ops_wait_ns();
    a.ntb = p.ntb;
    a.N = p.N;
    a.split = p.split;
    a.part = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + p.part_at);
    a.slots = (512 - 2 * a.N) / kTcSlotCols;
    if (a.slots > kTcMaxSlots)
        a.slots = kTcMaxSlots;
    // shared memory: 96 KiB of the tokens' blocks (what they take to come from
    // L2), six at most, the rest to the table
    const size_t fixed = 1024 + sizeof(Tc4Tail) + kSRing * kTcSBytes, bstage = (size_t)a.N * 256;
    a.bstages = (int)((96 << 10) / bstage);
    if (a.bstages > 6)
        a.bstages = 6;
    a.wstages = (int)((kTcSmem - fixed - a.bstages * bstage) / kTcWBytes);
    if (a.wstages > kTcMaxStages)
        a.wstages = kTcMaxStages;
    a.idesc = 1u << 4 | (uint32_t)(a.N >> 3) << 17 | (uint32_t)(2 * kTcRows >> 4) << 24;  // f32 += f16 f16, K-major
    CUtensorMap tm_w, tm_s, tm_x;
    if (!make_load_map(&tm_w, m.codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, (m.K + 1) / 2, m.V, m.ldc, kTcRows) ||
        !make_byte_map(&tm_s, m.gscales, (m.K + (1 << m.log_group) - 1) >> m.log_group, m.V, m.ldg, kTcSBox, kTcRows) ||
        !make_load_map(&tm_x, workspace, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, kp, m.T * parts, kp, a.N / 2))
        return cudaErrorInvalidValue;
    auto pick = [&](auto lg) {
        constexpr int LG = decltype(lg)::value;
        return m.obf16 ? (a.split > 1 ? k_mm4_tc<true, LG, false> : k_mm4_tc<false, LG, false>)
                       : (a.split > 1 ? k_mm4_tc<true, LG, true> : k_mm4_tc<false, LG, true>);
    };
    const auto kernel = m.log_group == 5   ? pick(std::integral_constant<int, 5>{})
                        : m.log_group == 6 ? pick(std::integral_constant<int, 6>{})
                                           : pick(std::integral_constant<int, 7>{});
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kTcSmem);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kTcThreads);
    cfg.dynamicSmemBytes = fixed + a.bstages * bstage + (size_t)a.wstages * kTcWBytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const int64_t tiles = (m.V + 2 * kTcRows - 1) / (2 * kTcRows) * a.ntb * a.split;
    cfg.gridDim = dim3(kSms);
    int fit = 0;
    e = cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg);
    if (e != cudaSuccess)
        return e;
    if (fit < 1)
        return cudaErrorInvalidConfiguration;
    cfg.gridDim = dim3((unsigned)(2 * (tiles < fit ? tiles : fit)));
    e = cudaLaunchKernelEx(&cfg, kernel, tm_w, tm_s, tm_x, a);
    if (e == cudaSuccess && a.split > 1)
        e = launch_k(k_mm4_join, dim3((unsigned)((m.V + 255) / 256), (unsigned)m.T), dim3(256), 0, stream, true, a);
    return e;
}

// Warps, ring and shared memory of k_mm4_few; stages = 0 where the columns leave
// no room for a ring.
FewPlan few_plan(const Mm4Args &a)
{
    FewPlan p{};
    const int kboxes = (a.K + kBoxK - 1) / kBoxK, cols = (int)a.T * (a.xf32 ? 2 : 1);
    p.xpitch = kboxes * kBoxK * 2 + 64;  // neighbouring columns in different halves of the banks
    p.join_at = ((size_t)cols * p.xpitch + 127) / 128 * 128;
    auto ring = [&](int warps) {
        p.ring_at = (p.join_at + (size_t)warps * kBoxRows * kFewCols * sizeof(float) + 1023) / 1024 * 1024;
        const size_t fixed = p.ring_at + 4096;  // alignment, and what is declared in the kernel
        const size_t stages = fixed < kFewSmem ? (kFewSmem - fixed) / ((size_t)warps * kBoxBytes) : 0;
        return stages < 2 ? 0 : stages > kFewMaxStages ? kFewMaxStages : (int)stages;
    };
    const int most = ring(kFewWarps) ? kFewWarps : kFewWarps / 2;
    if (!ring(most))
        return p;
    // The rounds that the SMs need for the tiles, each its boxes' time and about one
    // box's for the joining: us for 2^0 .. 2^4 warps a tile, 128256 x 8192: 107 / 108 /
    // 101 / 112 / 121; 32000 x 4096: 21.3 / 18.4 / 20.3 / 22.3 / 23.1; 10000 x 1000: 6.1 / 4.9 /
    // 4.5 / - / -.  Then no more tiles to a CTA than these rounds need.
    const int64_t tiles = (a.V + kBoxRows - 1) / kBoxRows;
    int64_t best = INT64_MAX;
    for (int l = 0; (1 << l) <= most && (1 << l) <= kboxes; ++l) {
        const int64_t rounds = (tiles + kSms * (most >> l) - 1) / (kSms * (most >> l));
        const int64_t cost = rounds * ((kboxes + (1 << l) - 1 >> l) + 1);
        if (cost < best) {
            best = cost;
            p.log_ks = l;
            p.warps = (int)((tiles + kSms * rounds - 1) / (kSms * rounds)) << l;
        }
    }
    p.stages = ring(p.warps);
    p.smem = p.ring_at + 1024 + (size_t)p.stages * p.warps * kBoxBytes;
    return p;
}

template <typename XT, int LG>
cudaError_t launch_few4(const Mm4Args &a, const FewPlan &p, unsigned *flags, cudaStream_t stream)
{
    const cudaError_t e =
        cudaFuncSetAttribute(k_mm4_few<XT, LG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem - 2048);
    if (e != cudaSuccess)
        return e;
    CUtensorMap tm;
    if (!make_load_map(&tm, a.codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, (a.K + 1) / 2, a.V, a.ldc, kBoxRows))
        return cudaErrorInvalidValue;
    const int64_t per = (int64_t)(p.warps >> p.log_ks) * kBoxRows, rounds = (a.V + per - 1) / per;
    return launch_k(k_mm4_few<XT, LG>, dim3((unsigned)(rounds < kSms ? rounds : kSms)), dim3(p.warps * 32), p.smem, stream,
                    true, tm, a, p, flags, ops_wait_ns());
}

cudaError_t launch_mm4(const Mm4Args &a, void *workspace, unsigned *flags, cudaStream_t stream)
{
    if (aligned(a.codes, 16) && a.ldc % 16 == 0 && aligned(a.gscales, 16) && a.ldg % 16 == 0) {
        // us of the warps' kernel / of tcgen05, bf16: 2 x 128256 x 8192 102 / 146, 5 tokens 130 /
        // 147, 8 139 / 148; 8 x 32000 x 4096 24.4 / 27.3, 8 x 50257 x 768 10.2 / 12.1
        if (a.T * (a.xf32 ? 2 : 1) <= kFewCols) {
            const FewPlan p = few_plan(a);
            auto go = [&](auto lg) {
                return a.xf32 ? launch_few4<float, decltype(lg)::value>(a, p, flags, stream)
                              : launch_few4<bf16_t, decltype(lg)::value>(a, p, flags, stream);
            };
            if (p.stages > 0)
                return a.log_group == 5   ? go(std::integral_constant<int, 5>{})
                       : a.log_group == 6 ? go(std::integral_constant<int, 6>{})
                                          : go(std::integral_constant<int, 7>{});
        }
        return launch_tc4(a, workspace, flags, stream);
    }
    const int64_t vb = (a.V + kGV - 1) / kGV, tb = (a.T + kGT - 1) / kGT;
    return launch_k(k_mm4_any, dim3((unsigned)(vb * tb)), dim3(256), 0, stream, true, a, (unsigned)vb);
}

}  // namespace
}  // namespace ember

using namespace ember;

extern "C" {

size_t ember_matmul_nibble_workspace_bytes(int64_t T, int64_t V, int64_t K, ember_wdtype xtype)
{
    if (T < 0 || V < 1 || K < 1 || T > kMaxMmRows / 2 || V > kMaxMmRows || K > kMaxRowCols || !dtype_ok(xtype))
        return 0;
    return tc4_plan(T > 0 ? T : 1, V, K, xtype == EMBER_F32).bytes;  // the tokens' fp16 parts, the parts of a split K
}

ember_status ember_matmul_nibble(const void *x, int64_t ldx, ember_wdtype xtype, const uint8_t *codes, int64_t ldc,
                                 const uint8_t *gscales, int64_t ldg, const float *scales, int64_t T, int64_t V,
                                 int64_t K, int group, void *out, int64_t ldo, ember_wdtype otype, void *workspace,
                                 size_t bytes, unsigned *status, void *stream)
{
    const int log_group = group == 32 ? 5 : group == 64 ? 6 : group == 128 ? 7 : 0;
    if (T < 0 || V < 1 || K < 1 || !log_group || ldx < K || ldc < (K + 1) / 2 || ldg < (K + group - 1) / group ||
        ldo < V || !codes || !gscales || !scales || !status)
        return EMBER_ERR_INVALID_ARG;
    if (T > 0 && (!x || !out))
        return EMBER_ERR_INVALID_ARG;
    if (!dtype_ok(xtype) || !dtype_ok(otype))
        return EMBER_ERR_DTYPE;
    if (T > kMaxMmRows / 2 || V > kMaxMmRows || K > kMaxRowCols || ldx > (int64_t(1) << 31) ||
        ldc > (int64_t(1) << 31) || ldg > (int64_t(1) << 31) || ldo > (int64_t(1) << 32))
        return EMBER_ERR_UNSUPPORTED;
    if (!aligned(x, elem_size(xtype)) || !aligned(scales, 4) || !aligned(out, elem_size(otype)) ||
        !aligned(status, 4) || !aligned(workspace, 16))
        return EMBER_ERR_ALIGNMENT;
    if (T == 0)
        return EMBER_OK;
    if (!workspace || bytes < ember_matmul_nibble_workspace_bytes(T, V, K, xtype))
        return EMBER_ERR_WORKSPACE;
    // 2^31 tiles of the smallest size are 1.4e14 logits: more than the GPU holds
    if ((V + kGV - 1) / kGV * ((T + kGT - 1) / kGT) > INT32_MAX)
        return EMBER_ERR_UNSUPPORTED;
    const Mm4Args a{x,   codes, gscales, scales, out, ldx, ldc, ldg, ldo, T, V, (int)K, log_group, xtype == EMBER_F32,
                    otype == EMBER_BF16};
    return launched(launch_mm4(a, workspace, status, (cudaStream_t)stream));
}

}  // extern "C"
