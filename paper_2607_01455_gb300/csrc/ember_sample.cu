// One token drawn from each row of logits, by temperature, top-k, top-p and
// min-p from a given uniform number.
//
//   w_v = exp((z_v - M) / a), M the row's largest logit, a the temperature;
//         weights below 2^-40 count as none
//   top-k: the first k logits (the larger first, the lower index first among equals)
//   top-p: of these the shortest prefix whose weights reach p of their sum
//   min-p: of these the ones with w >= m; the first always stays
//   the token is the first v, by index, at which the kept weights up to v exceed u
//   times their sum; its log-probability is log(w_v / sum)
//
// All three filters keep a prefix of the same order: what is kept is a smallest
// logit and, among those equal to it, a highest index.
//
// Where a sum crosses u times the total decides which token is drawn, and a
// vocabulary has 10^5 such borders: sums in fp32 would miss the right one now
// and then, differently for every order of summation.  So the weights are 64-bit
// integers, units of 2^-S, whose sums are exact, the same for every grouping:
// the result depends on nothing but the row.  A weight itself is good to about
// 2^-33 of its value (see Weigher) or to a unit, with errors of either sign.
//
// A row is read once from HBM and a few times from L2; a logit's weight takes some 22
// instructions a time.  Passes over a row: the largest logit, the kept weights' sums by
// warp, and the warp's share in which the draw falls; before the second, with a
// top-k, the number of logits by bins of their weight and the few of the bins that
// matter, from which one CTA draws at once; with a top-p alone two passes with
// weights, the second of which is the kept weights' own (nucleus()).  Bound by the
// instructions where rows are many (1024 x 128256 bf16: 184 us, 1.4 TB/s, the bytes
// alone 39 us; top-k 50 and top-p 0.9 205; top-p alone 470), by the barriers
// and the latency of the passes where they are few (1 x 128256: 10, 18 and 32 us).
#include "ember_rows.cuh"
#include "ember_tc.cuh"

#include <type_traits>

namespace ember {
namespace {

using namespace rows;
using tc::cluster_sync;

typedef unsigned long long u64;

constexpr int kCutOctaves = 40;

// Forms of the kernel: a row over a cluster of CTAs, a row per CTA, and a row per
// small CTA for short rows.
enum Form { kCluster, kSingle, kShort };
template <Form FORM>
struct Cfg {
    static constexpr bool alone = FORM != kCluster;
    static constexpr int threads = FORM == kShort ? 128 : 512, warps = threads / 32;
    // columns of the table of powers: 16 are one for each lane of half a warp
    static constexpr int columns = FORM == kShort ? 4 : 16;
    // bins of the order in a round, and per octave
    static constexpr int log_bins = FORM == kShort ? 9 : 11, bins = 1 << log_bins, log_octave = FORM == kShort ? 3 : 5;
    // of top-p's first pass: half as wide
    static constexpr int fine_octave = log_octave + 1, fine_bins = kCutOctaves << fine_octave;
    static constexpr int list = FORM == kShort ? 512 : FORM == kSingle ? 2048 : 1536;  // entries of a bin that are put in order at once
    // So many are drawn from by comparing each with each, more by selections.  us of the one /
    // the other for about 60, 115, 170, 225 and 430 entries: 1 x 128256 18 22 24 30 60 / 21 24 25 25
    // 25; 60 x 128256 26 32 38 49 114 / 29 36 37 37 40; 304 x 128256 60 66 71 81 149 / 62 69 71 72 76.
    static constexpr int few = 128;
    static constexpr int ctas = alone ? 1 : 16;  // of a cluster, at most
};
constexpr int kMaxCluster = 16;  // CTAs of a row (a non-portable cluster size past 8)
constexpr int64_t kMaxV = 1 << 19;
constexpr float kInf = __builtin_huge_valf();
constexpr float kMaxFloat = 0x1.fffffep127f;
constexpr double kLog2e = 1.4426950408889634074;
constexpr double kMaxTemperature = 0x1p100;

// What the temperature and min-p of a row come to, as pairs of floats (the
// second holds what the first is off by).
struct RowSet {
    float c1, c2;  // log2(e) / temperature (temperature 1 for 0)
    float d1, d2;  // how far below the largest logit weights are cut: 40 / c
    float b1, b2;  // how far above it min-p begins: temperature log(min_p), -inf without
};
struct SampleArgs {
    const void *z;
    const float *u;
    const float *temperature, *top_p, *min_p;  // per row, or nullptr and the number below
    const int32_t *top_k;
    double temperature1, top_p1, min_p1;
    int64_t top_k1;
    RowSet set;  // of the numbers
    int64_t *ids;
    float *logprobs;
    int64_t ldz, T;
    int V;
    int log_unit;  // S
};

// 2^(62 - j / 256), j < 256.
struct Powers {
    u64 t[256];
};
constexpr Powers make_powers()
{
    Powers p{};
    for (int j = 0; j < 256; ++j) {
        const double x = -j / 256.0 * 0.69314718055994530942;
        double term = 1.0, sum = 0.0;
        for (int n = 24; n >= 1; --n)  // the exponential's series, the small terms first
            sum = (sum + 1.0) * x / n;
        term += sum;
        p.t[j] = (u64)(term * 4611686018427387904.0);
    }
    return p;
}
__device__ const Powers kPowers = make_powers();

// The weight of a logit z as an integer, units of 2^-S:
//
//   t = (M - z) / a log2(e),  w = 2^-t = 2^-k 2^-g,  k = t rounded to 1/256
//
// M c and c = log2(e) / a are kept as pairs of floats; the fused operations
// lose nothing before g is formed (|g| < 2^-8, off by 2^-33 at most), since
// m1 - k is exact: both are multiples of one unit and their difference is below
// 2^24 of it.  2^-g - 1 is a cubic polynomial, rounded to 2^-38; the power 2^-k is a
// table's entry and a shift.  The last bit, which the shift has cut, is set: the
// middle of what was cut to the same integer, where cutting alone would take
// half a unit from each of 10^5 small weights.  Only for logits from the cut on.
// Where |M c| is large (low temperatures) logits are taken from M first: those
// whose weights count are then so near to M that the difference is exact.
struct Weigher {
    float z0, c1, c2, m1, m2, start, cut;
};
constexpr float kGrid = 49152.f;  // 1.5 * 2^15: numbers next to it are multiples of 1/256

__host__ __device__ __forceinline__ void pair_of(double x, float &hi, float &lo)
{
    hi = (float)x;
    lo = (float)(x - (double)hi);
}
__host__ __device__ __forceinline__ RowSet row_set(double temperature, double min_p)
{
    RowSet r;
    const double c = fmin(kLog2e / (temperature == 0.0 ? 1.0 : temperature), 1e37);
    pair_of(c, r.c1, r.c2);
    pair_of(kCutOctaves / c, r.d1, r.d2);
    r.b1 = r.b2 = 0.f;
    if (!(min_p > 0.0))
        r.b1 = -kInf;
    else if (min_p < 1.0)
        pair_of(temperature * log(min_p), r.b1, r.b2);
    return r;
}

// The smallest float that is at least x + b1 + b2, |b2| below half an ulp of b1.
__device__ __forceinline__ float from_above(float x, float b1, float b2)
{
    const float y = x + b1, v = y - x;
    const float rest = (x - (y - v)) + (b1 - v) + b2;  // the first two exact
    if (!(rest > 0.f))
        return y;
    const unsigned b = __float_as_uint(y);
    return y == 0.f ? __uint_as_float(1u) : __uint_as_float(b & 0x80000000u ? b - 1 : b + 1);
}

__device__ __forceinline__ Weigher make_weigher(float M, const RowSet &r, int S)
{
    Weigher w;
    float p = M * r.c1, lo = __fmaf_rn(M, r.c2, __fmaf_rn(M, r.c1, -p));
    const bool far = !(fabsf(p) <= 16000.f);
    w.z0 = far ? M : 0.f;
    p = far ? 0.f : p;
    lo = far ? 0.f : lo;
    w.c1 = r.c1;
    w.c2 = r.c2;
    // the unit: 2^-22 of a power of two above |M c| + 64, so at most 1/256
    const unsigned e = (__float_as_uint(fabsf(p) + 64.f) >> 23) + 1 - 22;
    const float big = __uint_as_float(e << 23) * 12582912.f;
    w.m1 = __fadd_rn(__fadd_rn(p, big), -big);
    w.m2 = (p - w.m1) + lo;
    w.start = kGrid + (float)(62 - S) + p;
    w.cut = fmaxf(from_above(M, -r.d1, -r.d2), -kMaxFloat);  // never -inf, which is masked
    return w;
}

// What a thread keeps of it: 62 - S octaves are in the grid already.
template <int COLUMNS>
struct Weight {
    Weigher k;
    float grid;
    uint32_t table;  // its column of the table in shared memory
    static constexpr unsigned line = COLUMNS * 8;
    // The grid's point of a logit, as bits: the octave in the second byte, the
    // table's index in the first.
    __device__ __forceinline__ unsigned place(float z) const
    {
        return __float_as_uint(__fmaf_rn(z - k.z0, -k.c1, k.start));
    }
    __device__ __forceinline__ u64 integer(unsigned b, float p, unsigned &lead) const
    {
        u64 v;
        asm("ld.shared.u64 %0, [%1];" : "=l"(v) : "r"(table + (b & 255u) * line));
        const int h = __mulhi((int)(v >> 32), __float2int_rn(p));  // 2^36 2^-(k - floor k) (2^-g - 1)
        long long y;
        asm("mad.wide.s32 %0, %1, %2, %3;" : "=l"(y) : "r"(h), "r"(1 << 26), "l"((long long)v));
        lead = (unsigned)(y >> 50);
        return (u64)y >> __byte_perm(b, 0, 0x4441) | 1u;  // by the second byte: below 64 where the weight counts
    }
    // The weights of two logits; the arithmetic of a pair is that of each.  Also
    // their places, and their leading bits: w in units of 2^(S - 12) over their
    // octave's power of two, so between 2^11 and 2^12.
    __device__ __forceinline__ void pair(float za, float zb, u64 &wa, u64 &wb) const
    {
        unsigned place[2], lead[2];
        pair(za, zb, wa, wb, place, lead);
    }
    __device__ __forceinline__ void pair(float za, float zb, u64 &wa, u64 &wb, unsigned (&place)[2], unsigned (&lead)[2]) const
    {
        auto both = [](float v) { return make2(v, v); };
        const f2 x = add2(make2(za, zb), both(-k.z0));
        const f2 r = fma2(x, both(-k.c1), both(k.start));
        const f2 a = fma2(add2(r, both(-grid)), both(-1.f), both(k.m1));
        const f2 g = add2(fma2(x, both(-k.c1), a), fma2(x, both(-k.c2), both(k.m2)));
        // 2^38 (2^-g - 1)
        constexpr double l = 0.69314718055994530942, one = 274877906944.0;
        constexpr float c1 = (float)(-l * one), c2 = (float)(l * l / 2 * one), c3 = (float)(-l * l * l / 6 * one);
        const f2 p = mul2(g, fma2(g, fma2(g, both(c3), both(c2)), both(c1)));
        float ra, rb, pa, pb;
        split2(r, ra, rb);
        split2(p, pa, pb);
        place[0] = __float_as_uint(ra);
        place[1] = __float_as_uint(rb);
        wa = integer(place[0], pa, lead[0]);
        wb = integer(place[1], pb, lead[1]);
    }
    __device__ __forceinline__ u64 operator()(float z) const
    {
        u64 a, b;
        pair(z, z, a, b);
        return a;
    }
    // The weight in fp32, in the same units, of a logit that counts: 2^(S - k) 2^-g.
    __device__ __forceinline__ float value(float z, int S) const
    {
        const float x = z - k.z0, n = __fmaf_rn(x, -k.c1, k.start) - grid;
        const float g = __fmaf_rn(x, -k.c1, k.m1 - n) + __fmaf_rn(x, -k.c2, k.m2);
        return exp2f((float)S - n - g);
    }
};

// A bin of the order: a part of an octave, ascending from the largest logit on.
template <int LOG_OCTAVE>
__device__ __forceinline__ int bin_of(unsigned place, int S)
{
    // rounding may put the largest one step before 0
    const int n = (int)((place & 0x3FFFu) >> (8 - LOG_OCTAVE)) - ((62 - S) << LOG_OCTAVE) + 1;
    return n < 0 ? 0 : n;
}
// A number whose order as an integer is that of the logits, descending; -0 as 0.
__device__ __forceinline__ unsigned key_of(float z)
{
    const unsigned b = __float_as_uint(z + 0.f);
    return b & 0x80000000u ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned key)
{
    return __uint_as_float(key & 0x80000000u ? key : ~key & 0x7FFFFFFFu);
}

// floor(f x) for 0 <= f < 1 (others are brought there), and ceil(f x) for 0 < f <= 1
__device__ __forceinline__ u64 scaled(double f, u64 x, bool up)
{
    if (!(f > 0.0))
        return 0;
    const u64 b = (u64)__double_as_longlong(f);
    const int e = (int)(b >> 52) - 1023;  // f = m 2^(e - 52)
    if (e >= 0)
        return up ? x : x - 1;
    if (e < -64)
        return up ? 1 : 0;
    const u64 m = (b & 0xFFFFFFFFFFFFFull) | 1ull << 52;
    const u64 hi = __umul64hi(m, x), lo = m * x;
    const int s = 52 - e;  // 53 .. 116
    u64 q, rest;
    if (s < 64) {
        q = hi << (64 - s) | lo >> s;
        rest = lo << (64 - s);
    } else if (s == 64) {
        q = hi;
        rest = lo;
    } else {
        q = hi >> (s - 64);
        rest = hi << (128 - s) | (lo != 0);
    }
    return q + (up && rest);
}

__device__ __forceinline__ u64 warp_sum(u64 x)
{
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1)
        x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ u64 warp_scan(u64 x, int lane)  // inclusive
{
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const u64 y = __shfl_up_sync(0xffffffffu, x, o);
        x += lane >= o ? y : 0;
    }
    return x;
}

__device__ __forceinline__ u64 load_remote(const u64 *p, uint32_t rank)
{
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(tc::mapa_rank(tc::smem_addr(p), rank)) : "memory");
    return v;
}
__device__ __forceinline__ unsigned load_remote(const unsigned *p, uint32_t rank)
{
    unsigned v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(tc::mapa_rank(tc::smem_addr(p), rank)) : "memory");
    return v;
}
__device__ __forceinline__ void store_remote(unsigned *p, uint32_t rank, unsigned v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(tc::mapa_rank(tc::smem_addr(p), rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void store_remote(u64 *p, uint32_t rank, u64 v)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(tc::mapa_rank(tc::smem_addr(p), rank)), "l"(v) : "memory");
}

template <Form FORM>
struct alignas(16) Shared {  // what follows it in shared memory starts on 16 bytes
    using C = Cfg<FORM>;
    u64 table[256][C::columns];
    // exchanged between the CTAs, by turns: a number per warp of each
    u64 sums[2][C::ctas][C::warps];
    float maxima[2][C::ctas][C::warps];
    u64 found[2];  // by one thread of the cluster, for all
    u64 part[C::warps];
    u64 base, upper, goal;
    int bin;
    // of a list: the range of the keys that come into question, and how many do
    u64 first[C::warps], last[C::warps];
    unsigned many[C::warps], picked;
    RowSet set[2];  // of this row and the next
};
struct Entry {
    float z;
    int v;
    u64 w;
};
// The sums by bin of one round, and what they become.
template <Form FORM>
union Bins {
    using C = Cfg<FORM>;
    unsigned hist[2][C::bins];  // the lower and the upper halves of sums
    u64 cum[C::bins > C::fine_bins ? C::bins : C::fine_bins];
    Entry all[C::alone ? 1 : C::list];  // the lists of all CTAs
};
template <Form FORM>
struct alignas(16) FilterShared {
    u64 coarse[2][32];  // of a round: the sums up to the end of each 32nd of the bins
    Bins<FORM> bins[Cfg<FORM>::alone ? 1 : 2];  // by turns: other CTAs read one round's sums while the next one's are formed
    Entry list[Cfg<FORM>::list];
    unsigned count;
};

// A CTA's part of a row, in 16-byte units, which are read where they are: from
// HBM in the first pass, from L1 or L2 in the others.
template <typename ZT>
struct Row {
    static constexpr int VE = 16 / sizeof(ZT);
    const ZT *z;  // the first unit
    int n;        // the number of units
    int v0;       // index of the first unit's first logit; below 0 where a row starts inside a unit
    int V;
    __device__ __forceinline__ uint4 raw(int u) const
    {
        const int v = v0 + u * VE;
        if (v >= 0 && v + VE <= V)
            return __ldg(reinterpret_cast<const uint4 *>(z) + u);
        return edge(z + u * VE, v, V);
    }
    // A unit that the row fills in part: -inf outside of it.
    static __device__ __forceinline__ uint4 edge(const ZT *z, int v, int V)
    {
        using Bits = std::conditional_t<sizeof(ZT) == 2, unsigned short, unsigned>;
        unsigned w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = sizeof(ZT) == 2 ? 0xFF80FF80u : 0xFF800000u;
#pragma unroll
            for (int h = 0; h < VE / 4; ++h) {
                const int e = k * (VE / 4) + h;
                if (v + e >= 0 && v + e < V) {
                    const unsigned x = reinterpret_cast<const Bits *>(z)[e];
                    w[k] = sizeof(ZT) == 4 ? x : h ? (w[k] & 0xFFFFu) | x << 16 : (w[k] & 0xFFFF0000u) | x;
                }
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ void unpack(const uint4 &r, float (&z)[VE])
    {
        const unsigned w[4] = {r.x, r.y, r.z, r.w};
        if constexpr (sizeof(ZT) == 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                z[2 * k] = dev::bf16_lo(w[k]);
                z[2 * k + 1] = dev::bf16_hi(w[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                z[k] = __uint_as_float(w[k]);
        }
    }
    __device__ __forceinline__ void unit(int u, float (&z)[VE]) const { unpack(raw(u), z); }
};

// What is kept: logits above zthr, and those equal to it up to the index ithr.
struct Keep {
    float zthr;
    int ithr;
    __device__ __forceinline__ bool operator()(float z, int v) const { return z > zthr || (z == zthr && v <= ithr); }
};

// The CTA's work on a row, with the exchanges between the CTAs.
template <typename ZT, Form FORM>
struct Draw {
    using K = Cfg<FORM>;
    static constexpr int VE = 16 / sizeof(ZT), kWarps = K::warps, kThreads = K::threads;
    Shared<FORM> *s;
    FilterShared<FORM> *f;
    Row<ZT> row;
    Weight<K::columns> weight;
    int ctas, rank, S, turn, round_turn, found_turn;
    int tid, lane, warp;

    __device__ __forceinline__ Bins<FORM> &sums_of(int turn) const { return f->bins[K::alone ? 0 : turn]; }
    // A warp has a contiguous share of the CTA's units.
    __device__ __forceinline__ int share() const { return (row.n + kWarps - 1) / kWarps; }
    // fn(z, v) for units of this thread, of logits z from index v on
    template <typename F>
    __device__ __forceinline__ void each_unit(F fn) const
    {
        const int m = share(), end = (warp + 1) * m < row.n ? (warp + 1) * m : row.n;
        int q = warp * m + lane;
        uint4 next = make_uint4(0, 0, 0, 0);
        if (q < end)
            next = row.raw(q);
        for (; q < end; q += 32) {
            float z[VE];
            row.unpack(next, z);
            if (q + 32 < end)  // a unit ahead
                next = row.raw(q + 32);
            fn(z, row.v0 + q * VE);
        }
    }
    __device__ __forceinline__ float largest() const
    {
        const int m = share(), end = (warp + 1) * m < row.n ? (warp + 1) * m : row.n;
        auto two = [](unsigned x) { return *reinterpret_cast<const __nv_bfloat162 *>(&x); };
        __nv_bfloat162 r2 = two(0xFF80FF80u);
        float r = -kInf;
#pragma unroll 4
        for (int q = warp * m + lane; q < end; q += 32) {
            const uint4 x = row.raw(q);
            if constexpr (VE == 8)
                r2 = __hmax2_nan(r2, __hmax2_nan(__hmax2_nan(two(x.x), two(x.y)), __hmax2_nan(two(x.z), two(x.w))));
            else
                r = max_nan(r, max_nan(max_nan(__uint_as_float(x.x), __uint_as_float(x.y)),
                                       max_nan(__uint_as_float(x.z), __uint_as_float(x.w))));
        }
        return VE == 8 ? max_nan(__low2float(r2), __high2float(r2)) : r;
    }
    // A unit's weights, those that are kept, added up.
    __device__ __forceinline__ u64 unit_sum(const Keep &keep, const float (&z)[VE], int v) const
    {
        u64 sum = 0;
#pragma unroll
        for (int e = 0; e < VE; e += 2) {
            u64 a, b;
            weight.pair(z[e], z[e + 1], a, b);
            if (keep(z[e], v + e))
                sum += a;
            if (keep(z[e + 1], v + e + 1))
                sum += b;
        }
        return sum;
    }
    __device__ __forceinline__ u64 kept_sum(const Keep &keep) const
    {
        u64 sum = 0;
        if (keep.ithr == INT32_MAX) {  // no logit is dropped for its index: one comparison each
            const float thr = keep.zthr;
            each_unit([&](const float(&z)[VE], int) {
#pragma unroll
                for (int e = 0; e < VE; e += 2) {
                    u64 a, b;
                    weight.pair(z[e], z[e + 1], a, b);
                    if (z[e] >= thr)
                        sum += a;
                    if (z[e + 1] >= thr)
                        sum += b;
                }
            });
        } else
            each_unit([&](const float(&z)[VE], int v) { sum += unit_sum(keep, z, v); });
        return sum;
    }

    // The sums over the CTAs of lower rank and over all, for every thread of the
    // cluster; those of this CTA's warps: s->sums[turn][rank].  put() before a
    // barrier of the row, got() behind it.
    __device__ __forceinline__ void put(u64 x)
    {
        turn ^= 1;
        x = warp_sum(x);
        if (K::alone ? lane == 0 : lane < ctas)
            store_remote(&s->sums[turn][rank][warp], lane, x);
    }
    __device__ __forceinline__ u64 got(u64 &before, u64 &total) const
    {
        if constexpr (K::alone) {
            before = total = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w)
                total += s->sums[turn][0][w];
            return total;
        }
        u64 lower = 0, own = 0, higher = 0;
        for (int i = lane; i < ctas * kWarps; i += 32) {
            const u64 y = (&s->sums[turn][0][0])[i];
            const int c = i / kWarps;
            lower += c < rank ? y : 0;
            own += c == rank ? y : 0;
            higher += c > rank ? y : 0;
        }
        before = warp_sum(lower);
        own = warp_sum(own);
        total = before + own + warp_sum(higher);
        return own;
    }
    __device__ __forceinline__ u64 exchange(u64 x, u64 &before, u64 &total)
    {
        put(x);
        row_sync();
        return got(before, total);
    }
    __device__ __forceinline__ void row_sync()
    {
        if constexpr (K::alone)
            __syncthreads();
        else
            cluster_sync();
    }
    // The CTA's sum of a value per thread.
    __device__ __forceinline__ u64 cta_sum(u64 x)
    {
        x = warp_sum(x);
        __syncthreads();
        if (lane == 0)
            s->part[warp] = x;
        __syncthreads();
        u64 t = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            t += s->part[w];
        return t;
    }
    // The first logit by index at which the sum of value(z, v) exceeds `target`,
    // found by this CTA after the exchange of the sums: done(z, v, value) by the
    // thread that has it.  sum_of(z, v) is that of a unit.
    template <typename U, typename F, typename G>
    __device__ __forceinline__ void locate(u64 target, U sum_of, F value, G done)
    {
        const u64 *part = s->sums[turn][rank];
        int w = 0;
        while (w + 1 < kWarps && target >= part[w])
            target -= part[w++];
        const int m = share(), first = w * m, end = first + m < row.n ? first + m : row.n;
        const int each = (m + kThreads - 1) / kThreads;  // units per thread, next to each other
        u64 sum = 0;
        for (int k = 0; k < each; ++k) {
            const int q = first + tid * each + k;
            if (q < end) {
                float z[VE];
                row.unit(q, z);
                sum += sum_of(z, row.v0 + q * VE);
            }
        }
        u64 upto = warp_scan(sum, lane);
        if (lane == 31)
            s->part[warp] = upto;
        __syncthreads();
        for (int k = 0; k < warp; ++k)
            upto += s->part[k];
        if (upto > target && upto - sum <= target) {
            s->upper = upto - sum;
            s->bin = tid;
        }
        __syncthreads();
        // the logits of that thread's units, one a lane and step
        if (warp == 0) {
            u64 at = s->upper;
            const int q0 = first + s->bin * each;
            for (int k = 0; k < each * VE; k += 32) {
                const int i = k + lane, q = q0 + i / VE;
                u64 x = 0;
                float z1 = 0.f;
                if (i < each * VE && q < end) {
                    float z[VE];
                    row.unit(q, z);
#pragma unroll
                    for (int e = 0; e < VE; ++e)
                        z1 = i % VE == e ? z[e] : z1;
                    x = value(z1, row.v0 + q * VE + i % VE);
                }
                const u64 sum_to = at + warp_scan(x, lane);
                if (sum_to > target && sum_to - x <= target)
                    done(z1, row.v0 + q * VE + i % VE, x);
                at = __shfl_sync(0xffffffffu, sum_to, 31);
            }
        }
        __syncthreads();  // the row and s->part have been read
    }
    // The log-probability of a logit of weight w among weights of the sum `total`.
    // The integer of a small weight has few bits (none to spare below 2^24 units, six
    // or four at the cut): there it is formed anew, good to 2^-20.
    __device__ __forceinline__ float log_share(float z, u64 w, u64 total) const
    {
        const float rest = (float)(total - w), all = (float)total;
        const float part = w < 1u << 24 ? weight.value(z, S) : (float)w;
        return 2 * w > total ? log1pf(-(rest / all)) : logf(part / all);
    }

    // The sum of a number over the CTAs.
    __device__ __forceinline__ u64 sum_at(const u64 *p, u64 base) const
    {
        if constexpr (K::alone)
            return base + *p;
        u64 y[K::ctas], g = base;  // all loads in flight at once
#pragma unroll
        for (int c = 0; c < K::ctas; ++c)
            y[c] = c < ctas ? load_remote(p, c) : 0;
#pragma unroll
        for (int c = 0; c < K::ctas; ++c)
            g += y[c];
        return g;
    }
    // The first bin at whose end `reached` holds of the sum (it stays so from there
    // on), with the sums before and behind it; -1 when it never does.  By a warp
    // whose lanes have the sums at the ends of their shares of the bins.
    template <int BINS, typename R>
    __device__ __forceinline__ int search(const Bins<FORM> &bins, u64 end, u64 base, R reached, u64 &low, u64 &high) const
    {
        constexpr int kShare = BINS / 32, kLane = (kShare + 31) / 32;  // bins of a share, and of a lane
        low = base;
        high = 0;
        unsigned reach = __ballot_sync(0xffffffffu, reached(end));
        if (!reach)
            return -1;
        const int q = __ffs(reach) - 1;
        const u64 prev = __shfl_sync(0xffffffffu, end, q > 0 ? q - 1 : 0);
        u64 g[kLane];
#pragma unroll
        for (int k = 0; k < kLane; ++k)  // the last lanes repeat the share's end
            g[k] = sum_at(bins.cum + q * kShare + min(lane * kLane + k, kShare - 1), base);
        reach = __ballot_sync(0xffffffffu, reached(g[kLane - 1]));
        const int r = __ffs(reach) - 1;
        u64 before = __shfl_sync(0xffffffffu, g[kLane - 1], r > 0 ? r - 1 : 0);
        before = r > 0 ? before : q > 0 ? prev : base;
        int found = 0;
        high = g[0];
#pragma unroll
        for (int k = 1; k < kLane; ++k)
            if (!reached(g[k - 1])) {
                found = k;
                low = g[k - 1];
                high = g[k];
            }
        found = __shfl_sync(0xffffffffu, found, r);
        low = __shfl_sync(0xffffffffu, low, r);
        high = __shfl_sync(0xffffffffu, high, r);
        low = found ? low : before;
        return q * kShare + r * kLane + found;
    }
    // cum and coarse of the bins from a thread's sums x of its own; hist has been
    // read when it comes back.  A barrier of the row follows.
    template <int N>
    __device__ __forceinline__ void cumulate(Bins<FORM> &bins, u64 *coarse, const u64 (&x)[N])
    {
        u64 sum = 0;
#pragma unroll
        for (int k = 0; k < N; ++k)
            sum += x[k];
        u64 upto = warp_scan(sum, lane);
        if (lane == 31)
            s->part[warp] = upto;
        __syncthreads();  // and hist has been read: cum takes its place
        upto -= sum;
        for (int w = 0; w < warp; ++w)
            upto += s->part[w];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            upto += x[k];
            bins.cum[tid * N + k] = upto;
        }
        constexpr int kShare = N * kThreads / 32;
        if ((tid + 1) * N % kShare == 0)
            coarse[tid * N / kShare] = upto;
    }

    // One round of the selection: the sums by digit of the order; the first digit
    // at which base and the sum up to it reach goal(base and all sums): returned
    // with base moved up to it and `upper` behind it, or -1 when nothing does.
    template <bool COUNT, typename D, typename T>
    __device__ __forceinline__ int round(const Keep &keep, D digit, T goal_of, u64 &base, u64 &upper, u64 &goal)
    {
        constexpr int kPer = K::bins / kThreads;  // bins per thread
        Bins<FORM> &bins = sums_of(round_turn);
        u64 *const coarse = f->coarse[round_turn];
        round_turn ^= 1;
        __syncthreads();
        for (int b = tid; b < (COUNT ? 1 : 2) * K::bins; b += kThreads)
            (&bins.hist[0][0])[b] = 0;
        __syncthreads();
        each_unit([&](const float(&z)[VE], int v) {
#pragma unroll
            for (int e = 0; e < VE; e += 2) {
                u64 w[2];
                if constexpr (!COUNT)
                    weight.pair(z[e], z[e + 1], w[0], w[1]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int d = keep(z[e + h], v + e + h) ? digit(z[e + h]) : -1;
                    if (d < 0)
                        continue;
                    if constexpr (COUNT)
                        atomicAdd(&bins.hist[0][d], 1u);
                    else {  // (64-bit ones are loops in shared memory)
                        const unsigned lo = (unsigned)w[h], old = atomicAdd(&bins.hist[0][d], lo);
                        const unsigned up = (unsigned)(w[h] >> 32) + (old + lo < lo);
                        if (up)
                            atomicAdd(&bins.hist[1][d], up);
                    }
                }
            }
        });
        __syncthreads();
        u64 x[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int b = tid * kPer + k;
            x[k] = bins.hist[0][b];
            if constexpr (!COUNT)
                x[k] += (u64)bins.hist[1][b] << 32;
        }
        cumulate(bins, coarse, x);
        row_sync();
        if (warp == 0) {
            const u64 end = sum_at(coarse + lane, base);
            goal = goal_of(__shfl_sync(0xffffffffu, end, 31));
            u64 low, high;
            const int found = search<K::bins>(bins, end, base, [&](u64 g) { return g >= goal; }, low, high);
            if (lane == 0) {
                s->bin = found;
                s->base = low;
                s->upper = high;
                s->goal = goal;
            }
        }
        __syncthreads();
        base = s->base;
        upper = s->upper;
        goal = s->goal;
        return s->bin;
    }
    __device__ __forceinline__ int bin(float z) const { return bin_of<K::log_octave>(weight.place(z), S); }

    // The place at which a bin begins.  Places are compared as they are: they grow
    // as the logits fall, past the cut too.
    template <int LOG_OCTAVE = K::log_octave>
    __device__ __forceinline__ unsigned place_from(int bin) const
    {
        constexpr unsigned kStart = 0x47400000u;  // 49152, the grid's first point
        return bin > 0 ? kStart + ((62u - S) << 8) + ((unsigned)(bin - 1) << (8 - LOG_OCTAVE)) : 0u;
    }

    // The kept logits of bins first .. last, with their weights (or 1), from all
    // CTAs: the number of them, and they themselves in *list unless there are more
    // than K::list.  `all`: for every CTA, or for the first alone.
    template <bool COUNT>
    __device__ __forceinline__ unsigned gather(const Keep &keep, int first, int last, bool all, Entry *&list)
    {
        if (tid == 0)
            f->count = 0;
        __syncthreads();
        auto take = [&](float z, int v) {
            const unsigned at = atomicAdd(&f->count, 1u);
            if (at < K::list) {
                f->list[at].z = z;
                f->list[at].v = v;
            }
        };
        const unsigned from = place_from(first), span = place_from(last + 1) - from;
        each_unit([&](const float(&z)[VE], int v) {
            bool in[VE], any = false;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                in[e] = weight.place(z[e]) - from < span;
                any |= in[e];
            }
            if (any)
#pragma unroll
                for (int e = 0; e < VE; ++e)
                    if (in[e] && keep(z[e], v + e))
                        take(z[e], v + e);
        });
        __syncthreads();
        for (unsigned i = tid; i < f->count && i < K::list; i += kThreads)
            f->list[i].w = COUNT ? 1 : weight(f->list[i].z);
        row_sync();
        return collect(all, list);
    }
    // The CTAs' lists as one, for every CTA or the first: see gather().
    __device__ __forceinline__ unsigned collect(bool all, Entry *&list)
    {
        if constexpr (K::alone) {
            list = f->list;
            return f->count;
        }
        list = sums_of(round_turn).all;  // the round before the last is over everywhere
        unsigned n = 0;
        if (all || rank == 0) {
            // lane c has CTA c's number, and the sum up to it
            const unsigned mine = lane < ctas ? load_remote(&f->count, lane) : 0;
            unsigned upto = mine;
#pragma unroll
            for (int o = 1; o < K::ctas; o *= 2) {
                const unsigned y = __shfl_up_sync(0xffffffffu, upto, o);
                upto += lane >= o ? y : 0;
            }
            n = __shfl_sync(0xffffffffu, upto, ctas - 1);
            if (n <= K::list)
                for (unsigned i0 = warp * 32; i0 < n; i0 += kThreads) {
                    const unsigned i = i0 + lane;
                    int c = 0;
                    unsigned begin = 0;
                    for (int k = 0; k + 1 < ctas; ++k) {
                        const unsigned end = __shfl_sync(0xffffffffu, upto, k);
                        if (i >= end) {
                            c = k + 1;
                            begin = end;
                        }
                    }
                    if (i < n) {
                        const u64 *p = reinterpret_cast<const u64 *>(&f->list[i - begin]);
                        u64 *q = reinterpret_cast<u64 *>(&list[i]);
                        const u64 x = load_remote(p, c), y = load_remote(p + 1, c);
                        q[0] = x;
                        q[1] = y;
                    }
                }
        }
        __syncthreads();
        return n;
    }

    // Of the entries of a list, in the order of their keys (no two are the same), the
    // first at which base and the sum of w up to it reach `goal`: sums by ranges of
    // keys, again and again, leave a few, which are compared with each other (lists up to
    // 512 with each other: 304 x 128256 with top-p 186 us, up to 128 160, up to 48 157).  By
    // one CTA.
    template <typename KEY, typename W>
    __device__ __forceinline__ unsigned select(const Entry *list, unsigned n, KEY key, W w, u64 base, u64 goal)
    {
        constexpr unsigned kAtOnce = 64;
        constexpr int kLog = FORM == kShort ? 7 : 9;
        static_assert(1 << kLog == kThreads && sizeof(Bins<FORM>) >= 4 * (3 * kThreads + kAtOnce), "a range per thread");
        unsigned *const hist = &sums_of(round_turn ^ 1).hist[0][0];  // the last round's sums have been read
        unsigned *const pick = hist + 3 * kThreads;
        const bool all = n <= kAtOnce;
        u64 lo = 0, hi = ~0ull;
        unsigned many = n;
        auto each_entry = [&](auto fn) {
            for (unsigned i = tid; i < n; i += kThreads) {
                const Entry e = list[i];
                const u64 k = key(e);
                if (k >= lo && k <= hi && w(e))
                    fn(i, k, w(e));
            }
        };
        while (!all) {
            u64 first = ~0ull, last = 0;
            many = 0;
            each_entry([&](unsigned, u64 k, u64) {
                first = min(first, k);
                last = max(last, k);
                ++many;
            });
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) {
                first = min(first, __shfl_xor_sync(0xffffffffu, first, o));
                last = max(last, __shfl_xor_sync(0xffffffffu, last, o));
            }
            many = __reduce_add_sync(0xffffffffu, many);
            if (lane == 0) {
                s->first[warp] = first;
                s->last[warp] = last;
                s->many[warp] = many;
            }
            for (int i = tid; i < 3 * kThreads; i += kThreads)
                hist[i] = 0;
            if (tid == 0)
                s->picked = 0;
            __syncthreads();
            many = 0;
#pragma unroll
            for (int q = 0; q < kWarps; ++q) {
                first = min(first, s->first[q]);
                last = max(last, s->last[q]);
                many += s->many[q];
            }
            if (many <= kAtOnce)
                break;
            const int bits = 64 - __clzll((long long)(last - first)), shift = bits > kLog ? bits - kLog : 0;
            each_entry([&](unsigned, u64 k, u64 x) {
                unsigned *const h = hist + (unsigned)((k - first) >> shift);
                atomicAdd(h, (unsigned)x & 0xFFFFu);
                atomicAdd(h + kThreads, (unsigned)(x >> 16) & 0xFFFFu);
                atomicAdd(h + 2 * kThreads, (unsigned)(x >> 32));
            });
            __syncthreads();
            const u64 x = hist[tid] + ((u64)hist[tid + kThreads] << 16) + ((u64)hist[tid + 2 * kThreads] << 32);
            u64 upto = warp_scan(x, lane);
            if (lane == 31)
                s->part[warp] = upto;
            __syncthreads();
            upto += base;
            for (int q = 0; q < warp; ++q)
                upto += s->part[q];
            if (upto >= goal && upto - x < goal) {
                s->bin = tid;
                s->base = upto - x;
            }
            __syncthreads();
            base = s->base;
            lo = first + ((u64)s->bin << shift);
            hi = lo + ((1ull << shift) - 1);
        }
        if (!all)
            each_entry([&](unsigned i, u64, u64) { pick[atomicAdd(&s->picked, 1u)] = i; });
        if (tid == 0)
            s->bin = 0;
        __syncthreads();
        for (unsigned i = warp; i < many; i += kWarps) {  // a warp per entry
            const unsigned at = all ? i : pick[i];
            const Entry e = list[at];
            u64 before = 0;
            for (unsigned j = lane; j < many; j += 32) {
                const Entry o = list[all ? j : pick[j]];
                before += key(o) < key(e) ? w(o) : 0;
            }
            before = base + warp_sum(before);
            if (before < goal && before + w(e) >= goal && lane == 0)
                s->bin = (int)at;
        }
        __syncthreads();
        return (unsigned)s->bin;
    }
    static __device__ __forceinline__ u64 order_key(const Entry &e) { return (u64)key_of(e.z) << 32 | (unsigned)e.v; }
    // The last one that is kept, from the list of those that come into question.
    __device__ __forceinline__ void order(Keep &keep, const Entry *list, unsigned n, u64 base, u64 goal)
    {
        const Entry e = list[select(list, n, order_key, [](const Entry &o) { return o.w; }, base, goal)];
        if constexpr (!K::alone)
            row_sync();  // the other CTAs have read this one's entries
        keep.zthr = e.z;
        keep.ithr = e.v;
    }

    // top-p.  One atomic addition per logit: of its weight's leading 12 bits (so that a
    // whole row's stay within 32), which give the sums by bin to 2^-10 of themselves,
    // from below but for a unit per logit, and so one or two bins for the cut.  A second pass adds up what is before these, exactly, and
    // collects their logits; with the cut among those known, the kept sums of the
    // warps are too, `mine` by thread, and no third pass is needed.  Returns
    // whether that is so: not where the bins have more logits than the list holds, nor
    // where min-p (zfloor) cuts before them, whatever their logits.
    __device__ __forceinline__ bool nucleus(Keep &keep, double top_p, float zfloor, u64 &mine)
    {
        constexpr int kBins = K::fine_bins, kPer = kBins / kThreads;
        Bins<FORM> &bins = sums_of(round_turn);
        u64 *const coarse = f->coarse[round_turn];
        round_turn ^= 1;
        __syncthreads();
        unsigned *const leads = &bins.hist[0][0];
        for (int b = tid; b < kBins; b += kThreads)
            leads[b] = 0;
        if (tid == 0)
            f->count = 0;
        __syncthreads();
        u64 sum = 0;
        each_unit([&](const float(&z)[VE], int v) {
#pragma unroll
            for (int e = 0; e < VE; e += 2) {
                u64 w[2];
                unsigned place[2], lead[2];
                weight.pair(z[e], z[e + 1], w[0], w[1], place, lead);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (keep(z[e + h], v + e + h)) {
                        sum += w[h];
                        atomicAdd(leads + min(bin_of<K::fine_octave>(place[h], S), kBins - 1), lead[h]);  // the last have a step of rounding too
                    }
            }
        });
        __syncthreads();
        u64 x[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int b = tid * kPer + k, up = S - 12 - ((b - 1) >> K::fine_octave);
            x[k] = up >= 0 ? (u64)leads[b] << up : (u64)leads[b] >> -up;
        }
        cumulate(bins, coarse, x);
        put(sum);
        row_sync();
        u64 before, mass;
        got(before, mass);
        u64 goal = scaled(top_p, mass, true);
        goal = goal > 0 ? goal : 1;
        if (warp == 0) {
            const u64 end = sum_at(coarse + lane, 0);
            u64 low, high;
            const int first = search<K::fine_bins>(bins, end, 0, [&](u64 g) { return g + (g >> 10) + kBins >= goal; }, low, high);
            // (below the unit a weight's leading bits exceed the weight, by less than one unit each)
            const int last = search<K::fine_bins>(bins, end, 0, [&](u64 g) { return g >= goal + (u64)row.V; }, low, high);
            if (lane == 0) {
                s->bin = first;
                s->base = (u64)(last < 0 ? kBins - 1 : last);
            }
        }
        __syncthreads();
        const int last = (int)s->base;  // the last bin has all that is behind it
        const unsigned from = place_from<K::fine_octave>(s->bin);
        const unsigned span = (last < kBins - 1 ? place_from<K::fine_octave>(last + 1) : ~0u) - from;
        if (weight.place(zfloor) < from)
            return false;  // min-p drops the cut's logit and all of its bin
        u64 above = 0;
        each_unit([&](const float(&z)[VE], int v) {
            bool in[VE], any = false;
#pragma unroll
            for (int e = 0; e < VE; e += 2) {
                u64 w[2];
                unsigned place[2], lead[2];
                weight.pair(z[e], z[e + 1], w[0], w[1], place, lead);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (place[h] < from)
                        above += w[h];
                    in[e + h] = place[h] - from < span;
                    any |= in[e + h];
                }
            }
            if (any)
#pragma unroll
                for (int e = 0; e < VE; ++e)
                    if (in[e] && keep(z[e], v + e)) {
                        const unsigned at = atomicAdd(&f->count, 1u);
                        if (at < K::list) {
                            f->list[at].z = z[e];
                            f->list[at].v = v + e;
                        }
                    }
        });
        __syncthreads();
        for (unsigned i = tid; i < f->count && i < K::list; i += kThreads)
            f->list[i].w = weight(f->list[i].z);
        put(above);
        row_sync();
        u64 base;
        got(before, base);
        Entry *list;
        const unsigned n = collect(true, list);
        if (n > K::list) {
            row_sync();  // the other CTAs have looked at this one's number
            u64 upper;
            const int q = round<false>(
                keep, [&](float z) { return bin(z); }, [&](u64) { return goal; }, base = 0, upper, goal);
            last_kept<false>(keep, q, base, goal);
            return false;
        }
        order(keep, list, n, base, goal);
        if (zfloor > keep.zthr)
            keep = {zfloor, INT32_MAX};
        // this CTA's logits of the list, to the warps that have them in their share
        mine = above;
        const int m = share() * VE;
        for (unsigned i = lane; i < f->count; i += 32) {
            const Entry e = f->list[i];
            if (keep(e.z, e.v) && (e.v - row.v0) / m == warp)
                mine += e.w;
        }
        return true;
    }

    // The logit of the order, in bin `first` with the sum `base` before it, at
    // which the sum (of the weights, or the number of logits) reaches `goal`
    // becomes the last one that is kept.
    template <bool COUNT>
    __device__ __forceinline__ void last_kept(Keep &keep, int first, u64 base, u64 goal)
    {
        Entry *list;
        const unsigned n = gather<COUNT>(keep, first, first, true, list);
        if (n <= K::list) {
            order(keep, list, n, base, goal);
            return;
        }
        u64 *slot = &s->found[found_turn];
        found_turn ^= 1;
        // too many: digits of the logits' bits down to one value
        unsigned known = 0, mask = 0;
        u64 upper;
        for (int top = 32; top > 0; top -= K::log_bins) {
            const int shift = top > K::log_bins ? top - K::log_bins : 0;
            const unsigned width = (1u << (top - shift)) - 1;
            const int d = round<COUNT>(
                keep,
                [&](float z) {
                    if (bin(z) != first)
                        return -1;
                    const unsigned k = key_of(z);
                    return (k & mask) == known ? (int)(k >> shift & width) : -1;
                },
                [&](u64) { return goal; }, base, upper, goal);
            known |= (unsigned)d << shift;
            mask |= width << shift;
        }
        const float z1 = value_of(known);
        const u64 w1 = COUNT ? 1 : weight(z1);
        const u64 ties = (goal - base + w1 - 1) / w1;  // so many of the logits equal to it are kept
        auto is = [&](float z, int v) { return (u64)(z == z1 && keep(z, v)); };
        auto unit = [&](const float(&z)[VE], int v) {
            u64 n1 = 0;
#pragma unroll
            for (int e = 0; e < VE; ++e)
                n1 += is(z[e], v + e);
            return n1;
        };
        u64 mine = 0, before, total;
        each_unit([&](const float(&z)[VE], int v) { mine += unit(z, v); });
        mine = exchange(mine, before, total);
        const u64 t = ties - 1;  // the first at which their number exceeds this
        if (before <= t && t < before + mine)
            locate(t - before, unit, is, [&](float, int v, u64) {
                for (int c = 0; c < ctas; ++c)
                    store_remote(slot, c, (u64)v);
            });
        row_sync();
        keep.zthr = z1;
        keep.ithr = (int)*slot;
    }

    // The whole draw from the n logits of a list that has the first k of the
    // order, by one CTA: of few, each compared with each.
    __device__ __forceinline__ void draw_from(Entry *list, unsigned n, u64 k, bool use_p, double top_p, float zfloor,
                                              float u, int64_t *id, float *logprob)
    {
        // what of the order is before each: a warp per entry, or eight lanes of it
        constexpr int G = FORM == kShort ? 8 : 32;
        const int sub = lane % G;
        u64 *const before = sums_of(round_turn ^ 1).cum;  // the last round's sums have been read
        u64 mass = 0;
        for (unsigned i0 = warp * (32 / G); i0 < n; i0 += kThreads / G) {  // the same for all lanes
            const unsigned i = i0 + lane / G;
            const Entry e = list[i < n ? i : 0];
            unsigned place = 0;
            u64 sum = 0;
            for (unsigned j = sub; j < n; j += G) {
                const Entry o = list[j];
                const bool earlier = o.z > e.z || (o.z == e.z && o.v < e.v);
                place += earlier;
                sum += earlier ? o.w : 0;
            }
#pragma unroll
            for (int o = G / 2; o >= 1; o >>= 1) {
                place += __shfl_xor_sync(0xffffffffu, place, o);
                sum += __shfl_xor_sync(0xffffffffu, sum, o);
            }
            if (sub == 0 && i < n) {
                before[i] = place < k ? sum : ~0ull;
                mass += place < k ? e.w : 0;
            }
        }
        mass = cta_sum(mass);
        const u64 goal = use_p ? scaled(top_p, mass, true) : ~0ull;
        u64 total = 0;
        for (unsigned i = tid; i < n; i += kThreads) {
            // the first of the order is always kept
            const bool in = before[i] == 0 || (before[i] < goal && list[i].z >= zfloor);
            if (!in)
                list[i].w = 0;
            total += list[i].w;
        }
        total = cta_sum(total);  // with a barrier: the list's weights are those kept
        const u64 at = scaled((double)u, total, false);
        for (unsigned i0 = warp * (32 / G); i0 < n; i0 += kThreads / G) {
            const unsigned i = i0 + lane / G;
            const Entry e = list[i < n ? i : 0];
            u64 sum = 0;
            for (unsigned j = sub; j < n; j += G)
                sum += list[j].v < e.v ? list[j].w : 0;
#pragma unroll
            for (int o = G / 2; o >= 1; o >>= 1)
                sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (sum <= at && at < sum + e.w && sub == 0 && i < n) {
                *id = e.v;
                *logprob = log_share(e.z, e.w, total);
            }
        }
    }
    // The same of many.
    __device__ __forceinline__ void draw_from_many(Entry *list, unsigned n, u64 k, bool use_p, double top_p, float zfloor,
                                                   float u, int64_t *id, float *logprob)
    {
        auto weight_of = [](const Entry &e) { return e.w; };
        // drops what is behind the entry or below the floor; the sum of the rest
        auto cut = [&](unsigned at, float floor) {
            const u64 last = order_key(list[at]);
            u64 sum = 0;
            for (unsigned i = tid; i < n; i += kThreads) {
                if (order_key(list[i]) > last || list[i].z < floor)
                    list[i].w = 0;
                sum += list[i].w;
            }
            return cta_sum(sum);
        };
        u64 total = cut(select(list, n, order_key, [](const Entry &) { return (u64)1; }, 0, k), use_p ? -kInf : zfloor);
        if (use_p) {
            const u64 goal = scaled(top_p, total, true);
            total = cut(select(list, n, order_key, weight_of, 0, goal > 0 ? goal : 1), zfloor);
        }
        const u64 at = scaled((double)u, total, false);
        const unsigned i = select(list, n, [](const Entry &e) { return (u64)(unsigned)e.v; }, weight_of, 0, at + 1);
        if (tid == 0) {
            *id = list[i].v;
            *logprob = log_share(list[i].z, list[i].w, total);
        }
    }
};

// CTAs per SM that the registers are shared out for.
constexpr int sample_ctas(bool filter, Form form) { return form == kShort ? (filter ? 6 : 8) : 2; }

// FILTER: calls with a top-k or a top-p.
template <typename ZT, bool FILTER, Form FORM>
__global__ void __launch_bounds__(Cfg<FORM>::threads, sample_ctas(FILTER, FORM)) k_sample(const SampleArgs a)
{
    constexpr int VE = 16 / sizeof(ZT), kThreads = Cfg<FORM>::threads, kWarps = Cfg<FORM>::warps;
    constexpr bool ALONE = Cfg<FORM>::alone;
    extern __shared__ __align__(16) unsigned char sample_smem[];
    Shared<FORM> *s = reinterpret_cast<Shared<FORM> *>(sample_smem);
    FilterShared<FORM> *f = reinterpret_cast<FilterShared<FORM> *>(sample_smem + sizeof(Shared<FORM>));
    Draw<ZT, FORM> d;
    d.s = s;
    d.f = f;
    d.ctas = ALONE ? 1 : (int)tc::cluster_count_in();
    d.rank = ALONE ? 0 : (int)tc::cluster_rank();
    d.S = a.log_unit;
    d.turn = d.round_turn = d.found_turn = 0;
    d.tid = threadIdx.x;
    d.lane = d.tid & 31;
    d.warp = d.tid >> 5;
    d.weight.grid = kGrid + (float)(62 - a.log_unit);
    d.weight.table = tc::smem_addr(&s->table[0][d.lane % Cfg<FORM>::columns]);
    d.row.V = a.V;
    const int rank = d.rank, tid = d.tid;
    const bool sets = a.temperature || a.min_p;  // a row's own

    for (int i = tid; i < 256 * Cfg<FORM>::columns; i += kThreads)
        (&s->table[0][0])[i] = kPowers.t[i / Cfg<FORM>::columns];
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    const int64_t step = ALONE ? gridDim.x : tc::cluster_count();
    for (int64_t t = ALONE ? blockIdx.x : tc::cluster_id(); t < a.T; t += step) {
        // where the row lies among the 16-byte units of its memory, and this CTA's
        const ZT *z = static_cast<const ZT *>(a.z) + t * a.ldz;
        const int skip = (int)((uintptr_t)z / sizeof(ZT) % VE);
        const int units = (skip + a.V + VE - 1) / VE;
        const int per = ALONE ? units : (units + d.ctas - 1) / d.ctas, u0 = rank * per;
        d.row.n = units - u0 < per ? (units > u0 ? units - u0 : 0) : per;
        d.row.v0 = u0 * VE - skip;
        d.row.z = z + d.row.v0;
        const double temp = a.temperature ? (double)a.temperature[t] : a.temperature1;
        const float u = a.u[t];
        const bool greedy = temp == 0.0;
        // read by all after the exchange; the last row's is not needed any more
        // once its own exchanges are over
        if (sets && tid == kThreads - 1)
            s->set[d.turn] = row_set(temp, a.min_p ? (double)a.min_p[t] : a.min_p1);
        const int set_at = d.turn;

        // the largest logit; a NaN is larger than all
        float m = warp_max_nan(d.largest());
        d.turn ^= 1;
        if (d.lane < d.ctas)
            store_remote(reinterpret_cast<unsigned *>(&s->maxima[d.turn][rank][d.warp]), d.lane, __float_as_uint(m));
        d.row_sync();
        for (int i = d.lane; i < d.ctas * kWarps; i += 32)
            m = max_nan(m, (&s->maxima[d.turn][0][0])[i]);
        m = warp_max_nan(m);

        const bool lost = !(m > -kInf && m < kInf) || !(temp >= 0.0 && temp <= kMaxTemperature);  // no distribution
        if (lost) {
            if (rank == 0 && tid == 0) {
                a.ids[t] = -1;
                a.logprobs[t] = __uint_as_float(0x7FC00000u);
            }
        } else {
            const RowSet set = sets ? s->set[set_at] : a.set;
            d.weight.k = make_weigher(m, set, a.log_unit);
            Keep keep{greedy ? m : d.weight.k.cut, INT32_MAX};
            // of the cut and of min-p
            const float zfloor = greedy ? m : fmaxf(keep.zthr, from_above(m, set.b1, set.b2));
            bool drawn = false, summed = false;
            u64 mine = 0;
            if constexpr (FILTER) {
                const double top_p = a.top_p ? (double)a.top_p[t] : a.top_p1;
                const int64_t top_k = a.top_k ? (int64_t)a.top_k[t] : a.top_k1;
                const bool use_p = !greedy && top_p < 1.0;
                auto bin = [&](float z) { return d.bin(z); };
                u64 base = 0, upper = 0, goal = 0;
                if (!greedy && top_k > 0 && top_k < a.V) {
                    const int q = d.template round<true>(keep, bin, [&](u64) { return (u64)top_k; }, base, upper, goal);
                    if (q >= 0 && upper <= Cfg<FORM>::list) {  // one CTA has them all and does the rest
                        Entry *list;
                        const unsigned n = d.template gather<false>(keep, 0, q, false, list);
                        if (rank == 0 && n <= Cfg<FORM>::few)
                            d.draw_from(list, n, (u64)top_k, use_p, top_p, zfloor, u, a.ids + t, a.logprobs + t);
                        else if (rank == 0)
                            d.draw_from_many(list, n, (u64)top_k, use_p, top_p, zfloor, u, a.ids + t, a.logprobs + t);
                        drawn = true;
                    } else if (q >= 0)
                        d.template last_kept<true>(keep, q, base, goal);
                }
                if (use_p && !drawn)
                    summed = d.nucleus(keep, top_p, zfloor, mine);
            }
            if (!drawn) {
                if (zfloor > keep.zthr)
                    keep = {zfloor, INT32_MAX};
                if (!summed)
                    mine = d.kept_sum(keep);
                u64 before, total;
                const u64 sum = d.exchange(mine, before, total);
                const u64 goal = greedy ? 0 : scaled((double)u, total, false);
                if (before <= goal && goal < before + sum)
                    d.locate(
                        goal - before, [&](const float(&x)[VE], int v) { return d.unit_sum(keep, x, v); },
                        [&](float x, int v) { return keep(x, v) ? d.weight(x) : (u64)0; },
                        [&](float x, int v, u64 w) {
                            a.ids[t] = v;
                            a.logprobs[t] = greedy ? 0.f : d.log_share(x, w, total);
                        });
            }
        }
    }
    if constexpr (!ALONE)
        cluster_sync();  // no CTA leaves while another may still read or write its memory
}

static_assert(sizeof(Shared<kCluster>) % 16 == 0 && sizeof(Shared<kSingle>) % 16 == 0 && sizeof(Shared<kShort>) % 16 == 0 &&
                  sizeof(Entry) == 16,
              "lists start on 16 bytes");

template <typename ZT, bool FILTER, Form FORM>
cudaError_t launch_form(const SampleArgs &a, int C, cudaStream_t stream)
{
    const auto kernel = k_sample<ZT, FILTER, FORM>;
    const size_t smem = sizeof(Shared<FORM>) + (FILTER ? sizeof(FilterShared<FORM>) : 0);
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess && C > 8)
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(Cfg<FORM>::threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)C;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cfg.gridDim = dim3((unsigned)(C * kSms));
    int fit = 0;
    e = cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg);
    if (e != cudaSuccess)
        return e;
    if (fit < 1)
        return cudaErrorInvalidConfiguration;
    const int64_t n = a.T < fit ? a.T : fit;
    cfg.gridDim = dim3((unsigned)(C * n));
    cfg.numAttrs = Cfg<FORM>::alone ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

// The form of a call, by what was measured (us without a filter / with top-k 50 and
// top-p 0.9 / with top-p 0.9 alone, bf16):
//   rows x logits     small CTA        CTA              cluster
//   1 x 1000          6.9  8.2  8.7    8.6  9.8  11.1   6.9  11.4 17.6
//   100 x 2048        7.8  10.1 9.3    7.4  10.2 11.9   7.2  12.0 17.9
//   152 x 8192        7.7  13.4 15.5   9.3  11.3 14.0   10.3 17.2 23.9
//   300 x 8192        8.8  14.4 16.5   9.6  14.7 18.9   10.4 16.5 23.5
//   1000 x 8192       19.4 28.8 40.9   30.0 47.7 60.0   32.1 56.3 79.1
//   1000 x 16384      32.8 39.5 68.7   38.5 55.4 84.2   40.9 63.0 101
//   300 x 16384       13.4 19.1 33.0   12.3 17.1 26.0   12.9 19.0 31.3
//   1000 x 32000      66.6 70.0 155    67.5 79.4 149    70.1 87.7 159
//   1 x 16384         10.4 16.7 22.5   8.3  12.4 16.4   8.1  13.9 21.0
//   1 x 32000         18.2 24.9 39.9   11.6 15.6 24.1   8.0  14.8 22.7
//   60 x 32000        18.3 25.9 53.5   11.9 16.2 27.0   11.9 18.9 28.5
//   60 x 64000        33.2 43.1 267    17.8 21.7 48.2   15.0 21.6 38.7
//   1 x 128256        -                29.2 31.7 77.7   9.8  17.6 32.3
//   152 x 128256      -                30.3 33.1 95.6   31.3 37.4 97.7
// So clusters are worth their barriers where they take 24576 logits and more off a CTA,
// and not as pairs.
constexpr int64_t kShortRow = 8192, kShareOut = 24576;
template <typename ZT, bool FILTER>
cudaError_t launch_sample(const SampleArgs &a, cudaStream_t stream)
{
    if (a.V <= (a.T > 2 * kSms ? 2 * kShortRow : a.T > kSms ? kShortRow : kShortRow / 4))
        return launch_form<ZT, FILTER, kShort>(a, 1, stream);
    // as many CTAs as keep the SMs busy, two each (of 16, 7 clusters run at once)
    int C = 1;
    while (C < kMaxCluster && a.T * C * 2 <= (C == 8 ? 7 * 16 : 2 * kSms))
        C *= 2;
    if (C > 2 && a.V - a.V / C >= kShareOut)
        return launch_form<ZT, FILTER, kCluster>(a, C, stream);
    return launch_form<ZT, FILTER, kSingle>(a, 1, stream);
}

}  // namespace
}  // namespace ember

using namespace ember;

extern "C" {

ember_status ember_sample(const void *logits, int64_t ldz, ember_wdtype ztype, const float *u, int64_t T, int64_t V,
                          double temperature, const float *temperatures, int64_t top_k, const int32_t *top_ks,
                          double top_p, const float *top_ps, double min_p, const float *min_ps, int64_t *ids,
                          float *logprobs, void *stream)
{
    if (T < 0 || V < 1 || ldz < V || (T > 0 && (!logits || !u || !ids || !logprobs)))
        return EMBER_ERR_INVALID_ARG;
    if (!temperatures && !(temperature >= 0.0 && temperature <= kMaxTemperature))
        return EMBER_ERR_INVALID_ARG;
    if ((!top_ks && top_k < 0) || (!top_ps && !(top_p > 0.0 && top_p <= 1.0)) ||
        (!min_ps && !(min_p >= 0.0 && min_p <= 1.0)))
        return EMBER_ERR_INVALID_ARG;
    if (!dtype_ok(ztype))
        return EMBER_ERR_DTYPE;
    if (T > INT32_MAX || V > kMaxV || ldz > (int64_t(1) << 32))
        return EMBER_ERR_UNSUPPORTED;
    if (!aligned(logits, elem_size(ztype)) || !aligned(u, 4) || !aligned(temperatures, 4) || !aligned(top_ks, 4) ||
        !aligned(top_ps, 4) || !aligned(min_ps, 4) || !aligned(ids, 8) || !aligned(logprobs, 4))
        return EMBER_ERR_ALIGNMENT;
    if (T == 0)
        return EMBER_OK;
    SampleArgs a{};
    a.z = logits;
    a.u = u;
    a.temperature = temperatures;
    a.top_k = top_ks;
    a.top_p = top_ps;
    a.min_p = min_ps;
    a.temperature1 = temperature;
    a.top_k1 = top_k;
    a.top_p1 = top_p;
    a.min_p1 = min_p;
    a.set = row_set(temperatures ? 1.0 : temperature, min_ps ? 0.0 : min_p);
    a.ids = ids;
    a.logprobs = logprobs;
    a.ldz = ldz;
    a.T = T;
    a.V = (int)V;
    // V weights of at most 2^S and a rounding's width stay below 2^64
    a.log_unit = 46;
    while (a.log_unit > 40 && (int64_t(1) << (63 - a.log_unit)) < V)
        --a.log_unit;
    const bool filter = top_ks || (top_k > 0 && top_k < V) || top_ps || top_p < 1.0;
    const cudaStream_t s = (cudaStream_t)stream;
    if (ztype == EMBER_BF16)
        return launched(filter ? launch_sample<bf16_t, true>(a, s) : launch_sample<bf16_t, false>(a, s));
    return launched(filter ? launch_sample<float, true>(a, s) : launch_sample<float, false>(a, s));
}

}  // extern "C"
