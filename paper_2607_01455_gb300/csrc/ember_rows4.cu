// Rows of a token table in 4 bits, and back.
//
//   r_v   the smallest power of two, at least 2^-126, with max_j |w_vj| <= 3136 r  (3136 = 7 * 448)
//   s_vg  max over the group of |w| / (7 r), rounded to e4m3
//   q_vj  w / (s r) rounded to an integer, kept within [-7, 7]; 0 where s is 0
//
// Both roundings are to nearest even of the quotient itself, not of its fp32
// value: r is a power of two, so w / r is exact, and what the division by 7 or
// by s cuts off is known from its remainder.
//
// The kernels pass once over their rows; bound by HBM on the way back, by HBM and the
// instructions on the way there.
#include "ember_quant4.cuh"

#include <type_traits>

namespace ember {
namespace {

using namespace rows;
using namespace quant4;

struct Rows4Args {
    const void *x;
    uint8_t *codes, *gscales;
    float *scales;
    int64_t ldx, ldc, ldg, V;
    int D, log_group;
    int words;  // whether codes take 8-byte stores
};

// The power of two of a row whose largest magnitude is `top` (finite, > 0), as
// its exponent.  3136 = 1.53125 * 2^11.
__device__ __forceinline__ int row_exponent(float top)
{
    const unsigned b = __float_as_uint(top);
    const int k = (int)(b >> 23) - 127 - 11 + ((b & 0x7FFFFFu) > 0x440000u);
    return k < -126 ? -126 : k;
}

// y / 7 (y >= 0) rounded to nearest even in e4m3.  The quotient to fp32 by a
// Newton step on a product with 1 / 7 (Markstein), moved off its place by one
// bit where the remainder says that it is not exact: no such number lies on a
// border between two e4m3 numbers that the quotient itself is not on.
__device__ __forceinline__ unsigned e4m3_of_seventh(float y)
{
    constexpr float seventh = 1.f / 7.f;
    const float q0 = y * seventh;
    const float q = __fmaf_rn(__fmaf_rn(-q0, 7.f, y), seventh, q0);
    const float rest = __fmaf_rn(-q, 7.f, y);
    const unsigned b = __float_as_uint(q) - (rest < 0.f);
    return __nv_cvt_float_to_fp8(__uint_as_float(rest == 0.f ? b : b | 1u), __NV_SATFINITE, __NV_E4M3);
}

// Eight values at any address, the first n of them (zeros behind): by the
// 16-byte units that hold them, moved by what the address is off one, where these
// lie between the matrix's first and last value; one by one otherwise.  The shift is
// the same for all units of a row.
template <typename XT>
__device__ __forceinline__ Raw<XT, 8> load_off(const XT *p, int n, const XT *begin, const XT *end)
{
    constexpr int W = sizeof(XT) == 2 ? 4 : 8;  // words of the values
    const int off = (int)((uintptr_t)p & 15);
    const uint4 *units = reinterpret_cast<const uint4 *>((uintptr_t)p - off);
    unsigned o[W];
    if (n >= 8 && (uintptr_t)units >= (uintptr_t)begin && (uintptr_t)(units + W / 4 + 1) <= (uintptr_t)end) {
        unsigned w[W + 4];
#pragma unroll
        for (int k = 0; k <= W / 4; ++k) {
            const uint4 v = __ldg(units + k);
            w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
        }
        const int bits = (off & 3) * 8;
        auto take = [&](auto first) {
            constexpr int f = decltype(first)::value;
#pragma unroll
            for (int k = 0; k < W; ++k)
                o[k] = sizeof(XT) == 2 ? __funnelshift_r(w[f + k], w[f + k + 1 < W + 4 ? f + k + 1 : W + 3], bits) : w[f + k];
        };
        switch (off >> 2) {
        case 0: take(std::integral_constant<int, 0>{}); break;
        case 1: take(std::integral_constant<int, 1>{}); break;
        case 2: take(std::integral_constant<int, 2>{}); break;
        default: take(std::integral_constant<int, 3>{}); break;
        }
    } else {
#pragma unroll
        for (int k = 0; k < W; ++k)
            o[k] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) {
                if constexpr (sizeof(XT) == 2)
                    o[e >> 1] |= (unsigned)p[e].u << (16 * (e & 1));
                else
                    o[e] = __float_as_uint(p[e]);
            }
    }
    Raw<XT, 8> r;
    if constexpr (sizeof(XT) == 2)
        r.v = make_uint4(o[0], o[1], o[2], o[3]);
    else {
        r.a = make_float4(__uint_as_float(o[0]), __uint_as_float(o[1]), __uint_as_float(o[2]), __uint_as_float(o[3]));
        r.b = make_float4(__uint_as_float(o[4]), __uint_as_float(o[5]), __uint_as_float(o[6]), __uint_as_float(o[7]));
    }
    return r;
}

// A row per TPR threads (a warp, or the CTA), kept in registers between its
// maximum and its codes: NU units of 16 values a thread, unit k of thread i
// being unit k TPR + i of the row.  What is done once per unit (the group's
// maximum by shuffles, its scale, addresses) is about as much as what is done
// for its values: 128256 x 8192 bf16 in units of 8 611 us, of 16 475 (5.6 TB/s; 82 %
// of the instruction slots taken), fp32 688 (6.9).  Rows off 16 bytes: 60000 x 2049 bf16
// 153 us (2.0 TB/s), fp32 215 (2.6).
template <typename XT, int TPR, int NU, bool GROUPED>
__global__ void __launch_bounds__(256) k_quantize4(Rows4Args a)
{
    __shared__ float part[8];
    const int lane = threadIdx.x & 31;
    const int i = TPR == 32 ? lane : (int)threadIdx.x;
    const int64_t row = TPR == 32 ? (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    if (TPR == 32 && row >= a.V)
        return;
    const XT *x = static_cast<const XT *>(a.x) + row * a.ldx;
    const XT *const x_end = static_cast<const XT *>(a.x) + (a.V - 1) * a.ldx + a.D;
    Raw<XT, 8> raw[NU][2];
#pragma unroll
    for (int k = 0; k < NU; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = (k * TPR + i) * 16 + h * 8;
            if constexpr (GROUPED)
                raw[k][h] = at < a.D ? load_raw<XT, 8>(x + at) : zero_raw<XT, 8>();
            else
                raw[k][h] = at < a.D ? load_off(x + at, a.D - at, static_cast<const XT *>(a.x), x_end) : zero_raw<XT, 8>();
        }
    float top[NU], whole = 0.f;
#pragma unroll
    for (int k = 0; k < NU; ++k) {
        if constexpr (sizeof(XT) == 2) {
            auto two = [](unsigned x) { return __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&x)); };
            auto four = [&](const uint4 &v) { return __hmax2_nan(__hmax2_nan(two(v.x), two(v.y)), __hmax2_nan(two(v.z), two(v.w))); };
            const __nv_bfloat162 m = __hmax2_nan(four(raw[k][0].v), four(raw[k][1].v));
            top[k] = max_nan(__low2float(m), __high2float(m));
        } else {
            top[k] = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float f[8];
                unpack<XT, 8>(raw[k][h], f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    top[k] = max_nan(top[k], fabsf(f[e]));
            }
        }
        whole = max_nan(whole, top[k]);
    }
    whole = warp_max_nan(whole);
    if constexpr (TPR > 32) {
        if (lane == 0)
            part[threadIdx.x >> 5] = whole;
        __syncthreads();
        whole = part[0];
#pragma unroll
        for (int w = 1; w < TPR / 32; ++w)
            whole = max_nan(whole, part[w]);
    }
    const bool live = whole > 0.f && whole < __builtin_huge_valf();
    const int ex = live ? row_exponent(whole) : 0;
    const float down = __uint_as_float((unsigned)(127 - ex) << 23);  // 1 / r
    if (i == 0)
        a.scales[row] = live ? __uint_as_float((unsigned)(ex + 127) << 23)
                             : whole == 0.f ? 0.f : __uint_as_float(0x7FC00000u);
    const int lanes = 1 << (a.log_group - 4);  // of a group: 2, 4 or 8
    uint8_t *codes = a.codes + row * a.ldc, *gscales = a.gscales + row * a.ldg;
    const f2 down2 = make2(down, down);
#pragma unroll
    for (int k = 0; k < NU; ++k) {
        const int u = k * TPR + i;
        if (k * TPR * 16 >= a.D)  // the same for all threads of a warp
            break;
        float g = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
        if (lanes > 2)
            g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
        if (lanes > 4)
            g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 4));
        unsigned byte = 0;
        float s = 0.f, inv = 0.f;
        if (live) {
            byte = e4m3_of_seventh(g * down);
            s = e4m3_value(byte);
            inv = s > 0.f ? __fdividef(1.f, s) : 0.f;  // and every quotient then 0
        }
        if (u * 16 < a.D && (lane & (lanes - 1)) == 0)
            gscales[u * 16 >> a.log_group] = (uint8_t)byte;
        // The quotients x / s to fp32, within [-7, 7] but for subnormal s (others are
        // rounded by a sixteenth at most).  That of a bf16 number is either on a
        // border between two integers or 2^-9 of itself away from it, and exact on
        // it; that of an fp32 number may round onto one, and the remainder says from
        // where.  A sum with 1.5 * 2^23 + 8 has q + 8 in its last bits.
        constexpr float magic = 12582912.f + 8.f;
        const f2 inv2 = make2(inv, inv), minus_s = make2(-s, -s), magic2 = make2(magic, magic);
        unsigned c[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float f[8];
            unpack<XT, 8>(raw[k][half], f);
            unsigned bits[8];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const f2 x2 = mul2(make2(f[e], f[e + 1]), down2);
                const f2 h0 = mul2(x2, inv2);
                f2 h = fma2(fma2(h0, minus_s, x2), inv2, h0);
                if (byte < 8u) {
                    float p, q;
                    split2(h, p, q);
                    h = make2(fminf(fmaxf(p, -7.f), 7.f), fminf(fmaxf(q, -7.f), 7.f));
                }
                float b[2];
                split2(add2(h, magic2), b[0], b[1]);
                if constexpr (sizeof(XT) == 4) {
                    float hs[2], xs[2];
                    split2(h, hs[0], hs[1]);
                    split2(x2, xs[0], xs[1]);
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const float d = hs[q] - __fadd_rn(b[q], -magic);
                        if (fabsf(d) == 0.5f && __fmaf_rn(-hs[q], s, xs[q]) * d > 0.f)
                            b[q] += 2.f * d;
                    }
                }
                bits[e] = __float_as_uint(b[0]);
                bits[e + 1] = __float_as_uint(b[1]);
            }
            // the last four bits of each, what is before them taken off at the end
            unsigned v = bits[7];
#pragma unroll
            for (int e = 6; e >= 0; --e)
                v = v * 16u + bits[e];
            c[half] = live ? v - 0x4B400000u * 0x11111111u : 0x88888888u;
        }
        if (a.words && u * 16 + 16 <= a.D)
            *reinterpret_cast<uint2 *>(codes + u * 8) = make_uint2(c[0], c[1]);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (u * 16 + 2 * e < a.D)
                    codes[u * 8 + e] = (uint8_t)(c[e >> 2] >> (8 * (e & 3)));
    }
}

template <typename XT, bool GROUPED>
cudaError_t launch_quantize4(const Rows4Args &a, cudaStream_t stream)
{
    const int units = (a.D + 15) / 16;
    auto go = [&](auto kernel, bool warps) {
        const unsigned n = (unsigned)(warps ? (a.V + 7) / 8 : a.V);
        return launch_k(kernel, dim3(n), dim3(256), 0, stream, true, a);
    };
    // A warp per row, without barriers, as long as its registers hold the row; us
    // of warps / CTAs, bf16: 200000 x 256 61 / 417, 131072 x 1024 66 / 270, 131072 x
    // 2048 117 / 268, 65536 x 4096 142 / 136.
    if (units <= 32)
        return go(k_quantize4<XT, 32, 1, GROUPED>, true);
    if (units <= 64)
        return go(k_quantize4<XT, 32, 2, GROUPED>, true);
    if (units <= 128)
        return go(k_quantize4<XT, 32, 4, GROUPED>, true);
    if (units <= 256)
        return go(k_quantize4<XT, 256, 1, GROUPED>, false);
    if (units <= 512)
        return go(k_quantize4<XT, 256, 2, GROUPED>, false);
    if (units <= 1024)
        return go(k_quantize4<XT, 256, 4, GROUPED>, false);
    return go(k_quantize4<XT, 256, 8, GROUPED>, false);
}

struct Back4Args {
    const uint8_t *codes, *gscales;
    const float *scales;
    const void *ids;
    void *y;
    unsigned *status;
    int64_t ldc, ldg, ldy, T, V;
    int D, log_group, ids64;
    int tpr;    // threads of a row
    int words;  // whether codes take 8-byte loads
};

constexpr int back_unit(size_t size) { return size == 4 ? 16 : 8; }

// Rows in the table's order or those of given ids: q s exact, its product with r
// rounded to fp32 (not at all where r is a power of two), then to bf16.  GROUPED:
// rows of the output start on 16 bytes (32 of fp32); a thread takes 16 or 8
// values per step.  Otherwise it takes eight at the output's 16-byte boundaries, whose codes
// begin inside a word and may lie in two groups; the row's first and last few go
// one by one.  128256 x 8192 bf16 430 us (6.2 TB/s; in units of 16 476), 16381 rows of
// 896 in fp32 10.7 us (6.3 TB/s), 60000 x 2049 bf16 100 us (3.1 TB/s).
template <typename YT, bool GROUPED>
__global__ void __launch_bounds__(256) k_dequantize4(Back4Args a)
{
    const int64_t t = (int64_t)blockIdx.x * (256 / a.tpr) + threadIdx.x / a.tpr;
    const int step = gridDim.y * a.tpr;
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    if (t >= a.T)
        return;
    int64_t row = t;
    if (a.ids)
        row = a.ids64 ? static_cast<const int64_t *>(a.ids)[t] : (int64_t)static_cast<const int32_t *>(a.ids)[t];
    const int first = blockIdx.y * a.tpr + threadIdx.x % a.tpr;
    const bool bad = row < 0 || row >= a.V;
    YT *y = static_cast<YT *>(a.y) + t * a.ldy;
    if (bad) {  // nothing of the table is read
        if (first == 0)
            atomicOr(a.status, kFlagIdRange);
        for (int j = first; j < a.D; j += step) {
            const float o[1] = {0.f};
            store_group<YT, 1>(y + j, o);
        }
        return;
    }
    const float r = a.scales[row];
    const uint8_t *codes = a.codes + row * a.ldc, *gscales = a.gscales + row * a.ldg;
    const int nb = (a.D + 1) / 2;
    // a word of codes; what is behind the row's bytes as zeros
    auto word = [&](int w) {
        if (a.words && w * 4 + 4 <= nb)
            return *reinterpret_cast<const unsigned *>(codes + w * 4);
        unsigned c = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (w * 4 + e < nb)
                c |= (unsigned)codes[w * 4 + e] << (8 * e);
        return c;
    };
    auto scale_at = [&](int j) { return __float2half2_rn(e4m3_value(gscales[j >> a.log_group])); };
    auto values = [&](unsigned c, const __half2 *s, int ns, float(&f)[8]) {  // q s exact in fp16
        unsigned w[4];
        eight_integers(c, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 q = __half22float2(__hmul2(*reinterpret_cast<const __half2 *>(&w[e]), s[ns == 1 ? 0 : e]));
            f[e] = q.x * r;
            f[e + 4] = q.y * r;
        }
    };
    if constexpr (GROUPED) {
        // units of 16 values for fp32, of 8 for bf16, whose stores are then 16 bytes
        // next to one another (128256 x 8192: 476 us, in units of 16 521)
        constexpr int N = back_unit(sizeof(YT)) / 8;
        using Word = std::conditional_t<N == 2, uint2, unsigned>;
        const int whole = a.words ? a.D / (8 * N) : 0;
        constexpr int B = 4 / N;  // units whose loads are in flight together
        int u = first;
        for (; u < whole; u += B * step) {
            Word c[B];
            unsigned s[B];
#pragma unroll
            for (int k = 0; k < B; ++k)
                if (u + k * step < whole) {
                    c[k] = *reinterpret_cast<const Word *>(codes + (u + k * step) * 4 * N);
                    s[k] = gscales[(u + k * step) * 8 * N >> a.log_group];
                }
#pragma unroll
            for (int k = 0; k < B; ++k)
                if (u + k * step < whole) {
                    const __half2 sk = __float2half2_rn(e4m3_value(s[k]));
#pragma unroll
                    for (int h = 0; h < N; ++h) {
                        float f[8];
                        values(reinterpret_cast<const unsigned *>(&c[k])[h], &sk, 1, f);
                        store_group<YT, 8>(y + ((u + k * step) * N + h) * 8, f);
                    }
                }
        }
        // the rest of a row: its first unit is this thread's if the count comes out so
        for (u = whole + (first - whole % step + step) % step; u * 8 * N < a.D; u += step) {
            const __half2 s = scale_at(u * 8 * N);
#pragma unroll
            for (int h = 0; h < N; ++h) {
                const int at = (u * N + h) * 8;
                float f[8];
                values(word(N * u + h), &s, 1, f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (at + e < a.D) {
                        const float o[1] = {f[e]};
                        store_group<YT, 1>(y + at + e, o);
                    }
            }
        }
    } else {
        constexpr int VE = 16 / sizeof(YT);
        const int skip = (int)((uintptr_t)y / sizeof(YT) % VE);
#pragma unroll 2
        for (int u = first; u * 8 - skip < a.D; u += step) {
            const int j = u * 8 - skip, j0 = j < 0 ? 0 : j, j1 = j + 7 < a.D ? j + 7 : a.D - 1;
            // floor(j / 8), with j >= -7
            const int w = j < 0 ? -1 : j >> 3;
            const unsigned lo = w < 0 ? 0 : word(w), hi = (j & 7) ? word(w + 1) : 0;
            const unsigned c = __funnelshift_r(lo, hi, (j & 7) * 4);
            const int edge = (((j0 >> a.log_group) + 1) << a.log_group) - j;  // values before it have the first scale
            const __half2 s0 = scale_at(j0), s1 = scale_at(j1);
            __half2 s[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s[e] = __halves2half2(e < edge ? __low2half(s0) : __low2half(s1), e + 4 < edge ? __low2half(s0) : __low2half(s1));
            float f[8];
            values(c, s, 4, f);
            if (j >= 0 && j + 8 <= a.D) {
                if constexpr (sizeof(YT) == 2)
                    store_group<YT, 8>(y + j, f);
                else {
                    *reinterpret_cast<float4 *>(y + j) = make_float4(f[0], f[1], f[2], f[3]);
                    *reinterpret_cast<float4 *>(y + j + 4) = make_float4(f[4], f[5], f[6], f[7]);
                }
            } else
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j + e >= 0 && j + e < a.D) {
                        const float o[1] = {f[e]};
                        store_group<YT, 1>(y + j + e, o);
                    }
        }
    }
}

int log_group_of(int group) { return group == 32 ? 5 : group == 64 ? 6 : group == 128 ? 7 : 0; }

// What both directions check of a table.
ember_status check_table(const void *codes, int64_t ldc, const void *gscales, int64_t ldg, const void *scales, int64_t V,
                         int64_t D, int group)
{
    if (V < 0 || D < 1 || !log_group_of(group) || ldc < (D + 1) / 2 || ldg < (D + group - 1) / group)
        return EMBER_ERR_INVALID_ARG;
    if (V > 0 && (!codes || !gscales || !scales))
        return EMBER_ERR_INVALID_ARG;
    if (V > INT32_MAX || D > kMaxRowCols || ldc > (int64_t(1) << 31) || ldg > (int64_t(1) << 31))
        return EMBER_ERR_UNSUPPORTED;
    return aligned(scales, 4) ? EMBER_OK : EMBER_ERR_ALIGNMENT;
}

}  // namespace
}  // namespace ember

using namespace ember;

extern "C" {

ember_status ember_quantize_rows_nibble(const void *x, int64_t ldx, ember_wdtype xtype, int64_t V, int64_t D, int group,
                                  uint8_t *codes, int64_t ldc, uint8_t *gscales, int64_t ldg, float *scales,
                                  void *stream)
{
    const ember_status st = check_table(codes, ldc, gscales, ldg, scales, V, D, group);
    if (st != EMBER_OK)
        return st;
    if (ldx < D || ldx > (int64_t(1) << 31) || (V > 0 && !x))
        return EMBER_ERR_INVALID_ARG;
    if (!dtype_ok(xtype))
        return EMBER_ERR_DTYPE;
    if (!aligned(x, elem_size(xtype)))
        return EMBER_ERR_ALIGNMENT;
    if (V == 0)
        return EMBER_OK;
    const Rows4Args a{x, codes, gscales, scales, ldx, ldc, ldg, V, (int)D, log_group_of(group),
                      aligned(codes, 8) && ldc % 8 == 0};
    const bool grouped8 = D % 8 == 0 && grouped(x, ldx, xtype);
    const cudaStream_t s = (cudaStream_t)stream;
    if (xtype == EMBER_BF16)
        return launched(grouped8 ? launch_quantize4<bf16_t, true>(a, s) : launch_quantize4<bf16_t, false>(a, s));
    return launched(grouped8 ? launch_quantize4<float, true>(a, s) : launch_quantize4<float, false>(a, s));
}

ember_status ember_dequantize_rows_nibble(const uint8_t *codes, int64_t ldc, const uint8_t *gscales, int64_t ldg,
                                    const float *scales, int64_t V, int64_t D, int group, const void *ids,
                                    ember_idtype idtype, int64_t T, void *y, int64_t ldy, ember_wdtype ytype,
                                    unsigned *status, void *stream)
{
    const ember_status st = check_table(codes, ldc, gscales, ldg, scales, V, D, group);
    if (st != EMBER_OK)
        return st;
    if (T < 0 || ldy < D || ldy > (int64_t(1) << 40) || (T > 0 && (!y || V < 1)) || (ids ? !status : T > V))
        return EMBER_ERR_INVALID_ARG;
    if (!dtype_ok(ytype) || (ids && idtype != EMBER_I32 && idtype != EMBER_I64))
        return EMBER_ERR_DTYPE;
    if (T > INT32_MAX)
        return EMBER_ERR_UNSUPPORTED;
    if (!aligned(y, elem_size(ytype)) || !aligned(ids, idtype == EMBER_I64 ? 8 : 4) || !aligned(status, 4))
        return EMBER_ERR_ALIGNMENT;
    if (T == 0)
        return EMBER_OK;
    Back4Args a{codes, gscales, scales, ids, y, status, ldc, ldg, ldy, T, V, (int)D, log_group_of(group),
                idtype == EMBER_I64, 32, aligned(codes, 8) && ldc % 8 == 0};
    const bool g8 = grouped(y, ldy, ytype);
    // 32 values a thread in a long call, a unit otherwise
    const int64_t unit = g8 ? back_unit(elem_size(ytype)) : 8, units = g8 ? (D + unit - 1) / unit : (D + 14) / 8;
    const int64_t per = T <= kSms ? 1 : 32 / unit;
    while (a.tpr < 256 && a.tpr * per < units)
        a.tpr *= 2;
    const int64_t rpc = 256 / a.tpr, cols = T <= kSms ? (units + a.tpr - 1) / a.tpr : 1;
    const dim3 grid((unsigned)((T + rpc - 1) / rpc), (unsigned)cols);
    auto go = [&](auto kernel) { return launched(launch_k(kernel, grid, dim3(256), 0, (cudaStream_t)stream, true, a)); };
    if (ytype == EMBER_BF16)
        return g8 ? go(k_dequantize4<bf16_t, true>) : go(k_dequantize4<bf16_t, false>);
    return g8 ? go(k_dequantize4<float, true>) : go(k_dequantize4<float, false>);
}

}  // extern "C"
