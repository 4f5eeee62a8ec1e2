// Softmax cross-entropy over the vocabulary with the gradient of the logits:
// the loss whose dlogits the LM-head step takes.
//
//   lse_t = log sum_v exp(z_tv),  nll_t = lse_t - z_t,y_t   (0 where ignored)
//   g_t = w_t / n (mean over the n counted tokens) or w_t (sum)
//   loss = sum_t g_t nll_t
//   dz_tv = g_t (exp(z_tv - lse_t) - [v = y_t])
//
// The statistics are a maximum and a sum in 32 bits: a thread keeps its own
// maximum and the sum of exp(z - maximum), and pairs (m, s), (m', s') join as
// (M, s e^(m-M) + s' e^(m'-M)), M = max(m, m').
//
// The pass is bound by HBM: each logit read once, each gradient written once.
// A row of up to 524288 logits is spread over a cluster of up to 16 CTAs and
// stays in their registers between the statistics and the gradient; the CTAs
// exchange one pair each through distributed shared memory.  4096 x 128256 bf16:
// 344 us, 6.12 TB/s, 0.90 of the copy bandwidth (from 1052 us reading each row
// twice); what is left is latency: 24 warps per SM of 64 logits a thread.
#include <atomic>

#include "ember_rows.cuh"
#include "ember_tc.cuh"

namespace ember {
namespace {

using namespace rows;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_huge_valf();

// 2^x within two ulps, results below 2^-126 as zero: they are less than one
// rounding of the row's sum, which is at least 1.
__device__ __forceinline__ float exp2_of(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// e^d of a difference: it is exact where it matters (near zero), so the
// rounding of d log2(e) costs a relative 2^-23 |d| at most.
__device__ __forceinline__ float exp_of(float d) { return exp2_of(d * kLog2e); }

struct MaxSum {
    float m, s;
};
// A maximum of -inf (nothing seen but -inf) is replaced by 0 in differences,
// so that exp gives 0 and not NaN.
__device__ __forceinline__ float finite_max(float m) { return m == -kInf ? 0.f : m; }
// The pairs of the lanes that differ in the bits below WIDTH (a power of two),
// joined: the maximum first, so that every sum is rescaled once.
template <int WIDTH>
__device__ __forceinline__ MaxSum lanes_join(MaxSum v)
{
    float m = v.m;
#pragma unroll
    for (int o = WIDTH / 2; o >= 1; o >>= 1)
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float s = v.s * exp_of(v.m - finite_max(m));
#pragma unroll
    for (int o = WIDTH / 2; o >= 1; o >>= 1)
        s += __shfl_xor_sync(0xffffffffu, s, o);
    return {m, s};
}

struct LossArgs {
    const void *z, *y;
    const float *w;
    void *d;
    float *nll, *loss;
    int *count;     // counted tokens, a part per CTA of the counting kernel
    double *total;  // parts of the loss
    int nparts;
    unsigned *status, *ticket;
    uint64_t wait_ns;
    int64_t ldz, ldd, T, V, ignore;
    int y64, mean;
};

__device__ __forceinline__ int64_t target_of(const LossArgs &a, int64_t t)
{
    return a.y64 ? static_cast<const int64_t *>(a.y)[t] : (int64_t)static_cast<const int32_t *>(a.y)[t];
}
// Whether token t counts; a target outside [0, V) that is not the ignored
// one does not, and is reported.
__device__ __forceinline__ bool counts(const LossArgs &a, int64_t y) { return y != a.ignore && y >= 0 && y < a.V; }

// The counted tokens of every kPartTokens or more.
constexpr int kMaxParts = 64;
constexpr int64_t kPartTokens = 2048;
__global__ void __launch_bounds__(1024) k_loss_count(LossArgs a)
{
    __shared__ int part[32];
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    int n = 0;
    bool bad = false;
    for (int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; t < a.T; t += (int64_t)gridDim.x * blockDim.x) {
        const int64_t y = target_of(a, t);
        n += counts(a, y);
        bad |= y != a.ignore && !counts(a, y);
    }
    if (bad)
        atomicOr(a.status, kFlagIdRange);
    n = __reduce_add_sync(0xffffffffu, n);
    if ((threadIdx.x & 31) == 0)
        part[threadIdx.x >> 5] = n;
    __syncthreads();
    if (threadIdx.x < 32) {
        n = __reduce_add_sync(0xffffffffu, part[threadIdx.x]);
        if (threadIdx.x == 0)
            a.count[blockIdx.x] = n;
    }
}
// Their number, by a whole warp.
__device__ __forceinline__ int counted(const LossArgs &a)
{
    int n = 0;
    for (int k = threadIdx.x & 31; k < a.nparts; k += 32)
        n += __ldcg(a.count + k);
    return __reduce_add_sync(0xffffffffu, n);
}

// The losses of tokens first, first + step, ... by thread, added in order, then
// a tree over the CTA; thread 0 gets the sum.  They were written by other
// CTAs: they are read through L2.
__device__ __forceinline__ double loss_sum(const LossArgs &a, int64_t first, int64_t step, double *part)
{
    double s = 0.0;
#pragma unroll 4
    for (int64_t t = first; t < a.T; t += step) {  // the loads of four tokens at once
        const int64_t y = target_of(a, t);
        const float nll = __ldcg(a.nll + t), w = a.w ? a.w[t] : 1.f;
        s += counts(a, y) ? (double)nll * (double)w : 0.0;
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1)
        s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0)
        part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int k = 0; k < (int)(blockDim.x >> 5); ++k)
            s += part[k];
    }
    return s;
}
__device__ __forceinline__ void write_loss(const LossArgs &a, double s, int n)
{
    *a.loss = n == 0 ? 0.f : (float)(a.mean ? s / (double)n : s);
}
// Whether this CTA is the last of the grid to come here, what the others have
// written then being visible; for every thread.
__device__ __forceinline__ bool last_cta(const LossArgs &a, int *flag)
{
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        *flag = atomicAdd(a.ticket, 1u) == gridDim.x - 1u;
        __threadfence();
        if (*flag)
            *a.ticket = 0;
    }
    __syncthreads();
    return *flag != 0;
}

// The total: a part per CTA, which the last one adds up in order.
__global__ void __launch_bounds__(512) k_loss_total(LossArgs a)
{
    __shared__ double part[16];
    __shared__ int last;
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    const double s = loss_sum(a, (int64_t)blockIdx.x * blockDim.x + threadIdx.x, (int64_t)gridDim.x * blockDim.x, part);
    if (threadIdx.x == 0)
        a.total[blockIdx.x] = s;
    if (last_cta(a, &last) && threadIdx.x < 32) {
        const int n = counted(a);
        double sum = 0.0;
        for (int k = 0; k < (int)gridDim.x; ++k)
            sum += __ldcg(a.total + k);
        if (threadIdx.x == 0)
            write_loss(a, sum, n);
    }
}

// One CTA per row, the row read twice (the second time from L2 when it is
// still there): for rows of any length, and for gradients whose rows start
// at other places of a 16-byte group than those of the logits.
template <typename ZT, typename DT, bool GRAD>
__global__ void __launch_bounds__(1024) k_loss_stream(LossArgs a)
{
    __shared__ MaxSum part[32];
    const int64_t t = blockIdx.x;
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    const int64_t y = target_of(a, t);
    DT *d = static_cast<DT *>(a.d) + t * a.ldd;
    if (!counts(a, y)) {
        if (GRAD)
            for (int64_t v = threadIdx.x; v < a.V; v += blockDim.x) {
                const float o[1] = {0.f};
                store_group<DT, 1>(d + v, o);
            }
        if (threadIdx.x == 0)
            a.nll[t] = 0.f;
        return;
    }
    const ZT *z = static_cast<const ZT *>(a.z) + t * a.ldz;
    float zy[1];
    unpack<ZT, 1>(load_raw<ZT, 1>(z + y), zy);
    MaxSum ms{-kInf, 0.f};
    for (int64_t v = threadIdx.x; v < a.V; v += blockDim.x) {
        float f[1];
        unpack<ZT, 1>(load_raw<ZT, 1>(z + v), f);
        const float m = fmaxf(ms.m, f[0]);
        if (m > ms.m)
            ms.s *= exp_of(ms.m - m);
        ms.m = m;
        ms.s += exp_of(f[0] - finite_max(m));
    }
    ms = lanes_join<32>(ms);
    if ((threadIdx.x & 31) == 0)
        part[threadIdx.x >> 5] = ms;
    __syncthreads();
    ms = lanes_join<32>(part[threadIdx.x & 31]);
    const float m = finite_max(ms.m);
    if (threadIdx.x == 0)
        a.nll[t] = ms.s == 0.f ? kInf : m - zy[0] + logf(ms.s);
    if (!GRAD)
        return;
    float g = a.w ? a.w[t] : 1.f;
    if (a.mean)
        g /= (float)counted(a);
    const float f = ms.s == 0.f ? 0.f : g / ms.s;
    const float hot = ms.s == 0.f ? 0.f : g;
    for (int64_t v = threadIdx.x; v < a.V; v += blockDim.x) {
        float o[1];
        unpack<ZT, 1>(load_raw<ZT, 1>(z + v), o);
        o[0] = exp_of(o[0] - m) * f;
        if (v == y)
            o[0] -= hot;
        store_group<DT, 1>(d + v, o);
    }
}

// Rows in the registers of a cluster.  Cluster q of n takes rows q, q + n,
// ...  A row is cut at the 16-byte units of its address (8 bf16 or 4 fp32
// logits); CTA `rank` has a contiguous slice of the units, which one bulk copy
// brings to its shared memory.  A thread takes up to 64 logits from there,
// finds their maximum and keeps e^(z - maximum) in registers: one exponential
// per logit, since the gradient is a multiple of it.  The buffer is then free:
// the copy of the cluster's next row runs while this one is reduced, exchanged
// and stored.  The CTAs exchange their pairs by asynchronous stores that
// complete on the receiver's mbarrier; a cluster barrier would wait, row by
// row, until the gradients stored before it had left the SM.  The logits
// before the first and after the last whole unit go one by one to threads of
// the first CTA.  The gradient's rows are at the same places of their units
// (launch_rows sees to it).
//
// A wait that gives up sets the timeout flag and ends its CTA's rows; the
// other CTAs of the cluster, which then lack its pairs, give up likewise.
template <typename T, int N>
__device__ __forceinline__ void unpack_unit(const uint4 &r, float (&f)[N])
{
    const unsigned u[4] = {r.x, r.y, r.z, r.w};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = dev::bf16_lo(u[k]);
            f[2 * k + 1] = dev::bf16_hi(u[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            f[k] = __uint_as_float(u[k]);
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_unit(T *p, const float (&f)[N])
{
    if constexpr (N == 8)
        store_group<T, 8>(p, f);
    else if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
    else
        *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
}

// Where the whole units of row t lie, and the slice of this CTA.
template <typename ZT>
struct Cut {
    static constexpr int VE = 16 / sizeof(ZT);
    int head, tail, units, per, u0, n;  // logits before and after the units; units per CTA; this CTA's units
    __device__ __forceinline__ Cut(const ZT *z, int V, int log_C, int rank)
    {
        head = (int)((VE - ((uintptr_t)z / sizeof(ZT)) % VE) % VE);
        head = head < V ? head : V;
        units = (V - head) / VE;
        tail = V - head - units * VE;
        per = (units + (1 << log_C) - 1) >> log_C;
        u0 = rank * per;
        n = units - u0 < per ? units - u0 : per;
        n = n > 0 ? n : 0;
    }
};

// The largest value of a unit (a NaN loses; it is found in the sum).
template <typename ZT>
__device__ __forceinline__ float unit_max(const uint4 &r)
{
    if constexpr (sizeof(ZT) == 2) {
        auto h = [](unsigned u) { return *reinterpret_cast<const __nv_bfloat162 *>(&u); };
        const __nv_bfloat162 m = __hmax2(__hmax2(h(r.x), h(r.y)), __hmax2(h(r.z), h(r.w)));
        return fmaxf(__low2float(m), __high2float(m));
    } else
        return fmaxf(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)),
                     fmaxf(__uint_as_float(r.z), __uint_as_float(r.w)));
}

constexpr int kPerThread = 64;  // logits of a row per thread
constexpr int kMaxClusterRow = 16;  // CTAs of a row (a non-portable cluster size past 8)
// Threads of a CTA: up to 256, several CTAs per SM; rows too long for 16 such
// CTAs take twice as many, up to 512.
constexpr int kRowThreads = 256;

// CTAs per SM that the registers are shared out for.  More warps hide more of
// a row's chain, until too much spills; us with one fewer / so many: 4096 x
// 50257 bf16 (224 threads) 180 / 156, 1024 x 252441 (256) 242 / 215, 2048 x
// 128256 187 / 182, 8192 x 32000 181 / 188.
// Rows of fp32 are nearer to the bandwidth and gain nothing, nor do calls of
// few tokens, which run once through.
constexpr int row_ctas(bool bf16, bool grad, bool here, int threads)
{
    return threads == 512   ? 1
           : threads == 256 ? (bf16 && !here ? 3 : 2)
           : threads == 224 ? (bf16 || !grad ? 3 : 2)
                            : (bf16 && !grad ? 6 : 4);
}

template <typename ZT, typename DT, bool GRAD, bool HERE, int MAXT>
__global__ void __launch_bounds__(MAXT, row_ctas(sizeof(ZT) == 2, GRAD, HERE, MAXT))
k_loss_rows(LossArgs a)
{
    constexpr int VE = Cut<ZT>::VE;
    constexpr int NU = kPerThread / VE;
    constexpr bool kKeepExp = GRAD;  // e^(z - m0) is kept
    extern __shared__ __align__(128) unsigned char buf[];  // this CTA's slice of a row
    __shared__ MaxSum part[32];
    __shared__ __align__(8) MaxSum all[2][kMaxClusterRow];
    __shared__ uint64_t full, joined[2];
    __shared__ int abort_;
    const int C = (int)tc::cluster_count_in(), rank = (int)tc::cluster_rank();
    const int log_C = __ffs(C) - 1;
    const int64_t first = blockIdx.x / C, step = gridDim.x / C;
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5, nwarps = nt >> 5;
    const int V = (int)a.V;
    const ZT *zbase = static_cast<const ZT *>(a.z);
    const uint32_t bar = tc::smem_addr(&full);
    volatile int *abort = &abort_;
    if (tid == 0) {
        tc::mbar_init(bar, 1);
        tc::mbar_init(tc::smem_addr(&joined[0]), 1);
        tc::mbar_init(tc::smem_addr(&joined[1]), 1);
        abort_ = 0;
        for (int k = 0; k < 2 * kMaxClusterRow; ++k)  // the places of CTAs that the cluster does not have stay so
            all[k / kMaxClusterRow][k % kMaxClusterRow] = {-kInf, 0.f};
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (C > 1)
        tc::cluster_arrive_release();  // waited for before the first store into another CTA: by then all are ready
    if constexpr (HERE) {  // otherwise the kernel before is k_loss_count, and only its result is waited for
        dev::grid_dep_wait();
        dev::grid_dep_launch();
    }

    // The copy of row t's slice, by thread 0; rows that do not count need none.
    uint32_t started = 0;
    auto start = [&](int64_t t, int64_t y) {
        const ZT *z = zbase + t * a.ldz;
        const Cut<ZT> q(z, V, log_C, rank);
        if (!counts(a, y) || q.n == 0)
            return;
        ++started;
        tc::mbar_expect_tx(bar, (uint32_t)q.n * 16);
        tc::bulk_load(tc::smem_addr(buf), z + q.head + (int64_t)q.u0 * VE, (uint32_t)q.n * 16, bar);
    };
    bool failed = false;  // a wait of this thread gave up
    bool met = false;     // the first cluster barrier is behind this CTA
    // A try may suspend its thread for longer than these copies take: a limit
    // below a microsecond is kept by looking once.
    auto wait = [&](uint32_t b, uint32_t parity) {
        if (!failed && !tc::mbar_look(b, parity) && (a.wait_ns < 1000 || !tc::mbar_spin(b, parity, abort, a.wait_ns))) {
            failed = true;
            atomicOr(a.status, kFlagTimeout);
            *abort = 1;
        }
    };
    int64_t y = target_of(a, first);
    int64_t ynext = first + step < a.T ? target_of(a, first + step) : 0;  // read a row ahead of its use
    if (tid == 0)
        start(first, y);
    // the number of counted tokens: from the kernel before, or, when the
    // tokens are few, from their targets at once
    float n = 1.f;
    if constexpr (HERE) {
        __shared__ int nvalid[32];
        int c = 0;
        bool bad = false;
#pragma unroll 4
        for (int64_t q = tid; q < a.T; q += nt) {
            const int64_t yq = target_of(a, q);
            c += counts(a, yq);
            bad |= yq != a.ignore && !counts(a, yq);
        }
        if (bad && blockIdx.x == 0)
            atomicOr(a.status, kFlagIdRange);
        c = __reduce_add_sync(0xffffffffu, c);
        if (lane == 0)
            nvalid[warp] = c;
        __syncthreads();
        c = 0;
        for (int k = 0; k < nwarps; ++k)
            c += nvalid[k];
        n = (float)c;
        if (blockIdx.x == 0 && tid == 0)
            *a.count = c;
    } else {
        dev::grid_dep_wait();
        dev::grid_dep_launch();
        if (a.mean)
            n = (float)counted(a);
        __syncthreads();  // the mbarriers are initialised
    }

    const float inv_n = a.mean ? 1.f / n : 1.f;  // infinite when no token counts, but then no row uses it
    // rows a whole number of units apart are all cut alike
    const bool alike = a.ldz % VE == 0;
    Cut<ZT> c(zbase, V, log_C, rank);
    uint32_t parity = 0;
    uint32_t round = 0;  // row number of this cluster: the exchange alternates between two buffers
    for (int64_t t = first; t < a.T; t += step, ++round) {
        const ZT *z = zbase + t * a.ldz;
        DT *d = static_cast<DT *>(a.d) + t * a.ldd;
        if (!alike)
            c = Cut<ZT>(z, V, log_C, rank);
        const bool on = counts(a, y);
        const bool more = t + step < a.T;
        const int64_t yafter = t + 2 * step < a.T ? target_of(a, t + 2 * step) : 0;
        const float w = a.w && on ? a.w[t] : 1.f;
        // the logit outside the units that this thread has, or -1
        int single = -1;
        if (rank == 0 && tid < c.head + c.tail)
            single = tid < c.head ? tid : V - c.tail + (tid - c.head);
        float zs = -kInf;
        if (on && single >= 0) {
            float f[1];
            unpack<ZT, 1>(load_raw<ZT, 1>(z + single), f);
            zs = f[0];
        }
        const int have = on ? c.n : 0;  // units in the buffer
        uint4 r[NU];
        if (have > 0) {
            wait(bar, parity);
            parity ^= 1u;
        }
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            // what is behind the slice counts as masked out
            constexpr unsigned fill = sizeof(ZT) == 2 ? 0xFF80FF80u : 0xFF800000u;
            if ((k + 1) * nt <= have)
                r[k] = reinterpret_cast<const uint4 *>(buf)[tid + k * nt];
            else
                r[k] = tid + k * nt < have ? reinterpret_cast<const uint4 *>(buf)[tid + k * nt]
                                           : make_uint4(fill, fill, fill, fill);
        }
        if (__syncthreads_or(failed))
            break;
        if (tid == 0 && more)
            start(t + step, ynext);

        float mt = zs;
#pragma unroll
        for (int k = 0; k < NU; ++k)
            mt = fmaxf(mt, unit_max<ZT>(r[k]));
        const float m0 = finite_max(mt);
        float kept[kKeepExp ? NU : 1][VE];  // e^(z - m0)
        const float es = exp_of(zs - m0);
        f2 sum = make2(es, 0.f), sum2 = make2(0.f, 0.f);
        const f2 minus = make2(-m0, -m0), scale = make2(kLog2e, kLog2e);
#pragma unroll
        for (int k = 0; k < NU; ++k) {
            float(&e)[VE] = kept[kKeepExp ? k : 0];
            unpack_unit<ZT, VE>(r[k], e);
#pragma unroll
            for (int q = 0; q < VE; q += 2) {
                const f2 x = mul2(add2(make2(e[q], e[q + 1]), minus), scale);
                split2(x, e[q], e[q + 1]);
                e[q] = exp2_of(e[q]);
                e[q + 1] = exp2_of(e[q + 1]);
                f2 &to = q & 2 ? sum2 : sum;
                to = add2(to, make2(e[q], e[q + 1]));
            }
        }
        MaxSum ms;
        ms.m = mt;
        {
            float x, y2;
            split2(add2(sum, sum2), x, y2);
            ms.s = x + y2;
        }
        ms = lanes_join<32>(ms);
        if (nwarps > 1) {
            if (lane == 0)
                part[warp] = ms;
            __syncthreads();
            ms = lanes_join<32>(lane < nwarps ? part[lane] : MaxSum{-kInf, 0.f});
        }
        if (C > 1) {
            if (round == 0)
                tc::cluster_wait();
            met = true;
            // every CTA's pair into every CTA
            const uint32_t p = round & 1u;
            const uint32_t jb = tc::smem_addr(&joined[p]);
            if (tid == 0)
                tc::mbar_expect_tx(jb, (uint32_t)C * sizeof(MaxSum));
            if (tid < C)
                tc::store_remote_async(&all[p][rank], tid, ms.m, ms.s, jb);
            wait(jb, round >> 1 & 1u);
            ms = lanes_join<kMaxClusterRow>(all[p][lane & (kMaxClusterRow - 1)]);
        }
        const float m = finite_max(ms.m);
        const bool live = on && ms.s != 0.f;
        if (!on && rank == 0 && tid == 0)
            a.nll[t] = 0.f;
        const float g = w * inv_n;
        const float gs = __fdividef(g, ms.s);  // a sum is between 1 and 2^19: within two ulps
        // by the thread's own maximum, not m0: where it saw nothing but -inf, its values
        // are 0 and so is the factor, which 0 - m could make infinite
        const float f = live ? exp_of(mt - m) * gs : 0.f;
        // the target's loss and gradient, by the thread that has it among its logits
        const int yu = on ? (int)y - c.head - c.u0 * VE : -1;  // its place among this slice's logits
        const bool mine = yu >= 0 && yu < c.n * VE && yu / VE % nt == tid;
        float hot = 0.f;
        if (mine) {
            // read again from the row: the copy's buffer may hold the next one already
            float zy[1];
            unpack<ZT, 1>(load_raw<ZT, 1>(z + y), zy);
            a.nll[t] = live ? (m - zy[0]) + logf(ms.s) : kInf;
            hot = live ? exp_of(zy[0] - m) * gs - g : 0.f;
        }
        if (single >= 0 && on && single == (int)y)
            a.nll[t] = live ? (m - zs) + logf(ms.s) : kInf;
        if constexpr (GRAD) {
            // a row that does not count, or is -inf throughout, has only zeros
            const f2 ff = make2(f, f);
#pragma unroll
            for (int k = 0; k < NU; ++k) {
                const int u = tid + k * nt;
                float(&e)[VE] = kept[k];
#pragma unroll
                for (int q = 0; q < VE; q += 2)
                    split2(mul2(make2(e[q], e[q + 1]), ff), e[q], e[q + 1]);
                if (u < c.n)
                    store_unit<DT, VE>(d + c.head + (int64_t)(c.u0 + u) * VE, e);
            }
            if (mine) {
                const float o[1] = {hot};
                store_group<DT, 1>(d + y, o);
            }
            if (single >= 0) {
                const float o[1] = {live ? exp_of(zs - m) * gs - (single == (int)y ? g : 0.f) : 0.f};
                store_group<DT, 1>(d + single, o);
            }
        }
        y = ynext;
        ynext = yafter;
    }
    const bool gave_up = __syncthreads_or(failed);
    if (C > 1 && !met)
        tc::cluster_wait();
    if (gave_up && tid == 0 && started)  // the copy it started last has landed before the CTA ends
        tc::mbar_wait_final(bar, (started - 1u) & 1u);
    // few tokens: the last CTA to come here adds the losses up
    if constexpr (HERE) {
        __shared__ double dpart[16];
        __shared__ int last;
        if (last_cta(a, &last)) {
            const double sum = loss_sum(a, tid, nt, dpart);
            if (tid == 0)
                write_loss(a, sum, __ldcg(a.count));
        }
    }
    if (C > 1)
        tc::cluster_sync();  // no CTA leaves while another may still send to it
    // What a CTA that gave up did not wait for may still be on its way to it; all of
    // it has been sent by now and takes about a microsecond.
    if (gave_up && tid == 0) {
        const uint64_t t0 = dev::now_ns();
        while (dev::now_ns() - t0 < 100000)
            ;
    }
}

// Threads per CTA and CTAs per row for rows of V logits; C = 0 where a row
// does not fit the registers of a cluster.
struct RowPlan {
    int C, nt;
    size_t smem;
};
// Up to so many tokens are one launch: every CTA counts the targets itself and
// the last one adds up the losses (127 x 50257 fp32: 18.2 us, with launches of
// their own for both 21.6; 1000 x 8000 bf16 16.5 and 16.9, 2000 x 8000 fp32 34
// and 32).  More would keep a CTA busy for longer than the launches take.
constexpr int64_t kFewRowsHere = 1024;
// So would more than these per thread of a CTA, short rows having small ones
// (one warp, 1000 fp32: 400 rows 9.9 us, with the launches 11.3; 500 rows 12.5
// and 11.7).
constexpr int64_t kFewPerThread = 12;

RowPlan row_plan(int64_t T, int64_t V, int esize)
{
    RowPlan p{0, 0, 0};
    const int64_t units = V / (16 / esize) + 1, nu = kPerThread / (16 / esize);
    int C = 1;
    while (C < kMaxClusterRow && units > C * kRowThreads * nu)
        C *= 2;
    const int64_t per = (units + C - 1) / C;
    if (per > 512 * nu || T * C > INT32_MAX)
        return p;
    p.C = C;
    p.nt = (int)((per + nu - 1) / nu + 31) / 32 * 32;
    p.smem = (size_t)per * 16;
    return p;
}

// As many clusters as run at once, each with a share of the rows; one per row
// when there are few.
template <typename K>
cudaError_t launch_cluster(K kernel, const LossArgs &a, const RowPlan &p, cudaStream_t stream)
{
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 << 10);
    if (e == cudaSuccess && p.C > 8)
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.T * p.C));
    cfg.blockDim = dim3(p.nt);
    cfg.dynamicSmemBytes = p.smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.C;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (a.T * p.C > kSms) {
        cfg.numAttrs = 1;
        int fit = 0;
        e = cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg);
        if (e != cudaSuccess)
            return e;
        if (fit < 1)
            return cudaErrorInvalidConfiguration;
        // Clusters that share the rows are as many as an empty GPU holds, so
        // they start on an empty one: let in while an earlier kernel still has
        // an SM or two, they are placed around it, and one that then finds no
        // room runs after all the others (4096 x 50257 bf16 295 us, 178 so).
        if (a.T > fit)
            cfg.gridDim = dim3((unsigned)fit * p.C);
        else
            cfg.numAttrs = 2;
    }
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename ZT, typename DT, bool GRAD>
cudaError_t launch_rows(LossArgs a, cudaStream_t stream)
{
    RowPlan p = row_plan(a.T, a.V, sizeof(ZT));
    constexpr int VE = 16 / sizeof(ZT);
    if (GRAD && (((uintptr_t)a.z / sizeof(ZT) - (uintptr_t)a.d / sizeof(DT)) % VE != 0 || (a.ldz - a.ldd) % VE != 0))
        p.C = 0;
    const bool here = p.C > 0 && a.T <= kFewRowsHere && a.T <= kFewPerThread * p.nt;
    a.nparts = here ? 1 : (int)(a.T / kPartTokens < kMaxParts ? a.T / kPartTokens + 1 : kMaxParts);
    cudaError_t e = cudaSuccess;
    if (!here)
        e = launch_k(k_loss_count, dim3(a.nparts), dim3(1024), 0, stream, true, a);
    if (e != cudaSuccess)
        return e;
    if (p.C == 0) {
        e = launch_k(k_loss_stream<ZT, DT, GRAD>, dim3((unsigned)a.T), dim3(1024), 0, stream, true, a);
        return e == cudaSuccess ? launch_k(k_loss_total, dim3(a.nparts), dim3(512), 0, stream, true, a) : e;
    }
    if (here)
        return p.nt <= 256 ? launch_cluster(k_loss_rows<ZT, DT, GRAD, true, 256>, a, p, stream)
                           : launch_cluster(k_loss_rows<ZT, DT, GRAD, true, 512>, a, p, stream);
    if (p.nt <= 128)
        e = launch_cluster(k_loss_rows<ZT, DT, GRAD, false, 128>, a, p, stream);
    else if (p.nt <= 224)
        e = launch_cluster(k_loss_rows<ZT, DT, GRAD, false, 224>, a, p, stream);
    else if (p.nt <= 256)
        e = launch_cluster(k_loss_rows<ZT, DT, GRAD, false, 256>, a, p, stream);
    else
        e = launch_cluster(k_loss_rows<ZT, DT, GRAD, false, 512>, a, p, stream);
    if (e == cudaSuccess)
        e = launch_k(k_loss_total, dim3(a.nparts), dim3(512), 0, stream, true, a);
    return e;
}

}  // namespace
}  // namespace ember

using namespace ember;

static std::atomic<uint64_t> ops_wait{kDefaultWaitNs};
uint64_t ember::ops_wait_ns() { return ops_wait.load(std::memory_order_relaxed); }

extern "C" {

size_t ember_softmax_loss_workspace_bytes(int64_t T)
{
    return T >= 0 && T <= INT32_MAX ? kMaxParts * (sizeof(double) + sizeof(int)) : 0;
}

ember_status ember_softmax_loss(const void *logits, int64_t ldz, ember_wdtype ztype, const void *targets,
                                ember_idtype idtype, const float *weights, int64_t ignore_index, int mean, int64_t T,
                                int64_t V, float *loss, float *nll, void *dlogits, int64_t ldd, ember_wdtype dtype,
                                void *workspace, size_t bytes, unsigned *status, void *stream)
{
    if (!loss || !status || T < 0 || V < 1 || ldz < V || (dlogits && ldd < V) || (mean != 0 && mean != 1))
        return EMBER_ERR_INVALID_ARG;
    if (T > 0 && (!logits || !targets || !nll || ldz > (int64_t(1) << 61) / T || (dlogits && ldd > (int64_t(1) << 61) / T)))
        return EMBER_ERR_INVALID_ARG;
    if (!dtype_ok(ztype) || (dlogits && !dtype_ok(dtype)) || (idtype != EMBER_I32 && idtype != EMBER_I64))
        return EMBER_ERR_DTYPE;
    if (T > INT32_MAX || V > INT32_MAX)
        return EMBER_ERR_UNSUPPORTED;
    if (!aligned(logits, elem_size(ztype)) || !aligned(targets, idtype == EMBER_I64 ? 8 : 4) || !aligned(weights, 4) ||
        !aligned(loss, 4) || !aligned(nll, 4) || !aligned(status, 4) || !aligned(workspace, 16) ||
        (dlogits && !aligned(dlogits, elem_size(dtype))))
        return EMBER_ERR_ALIGNMENT;
    if (!workspace || bytes < ember_softmax_loss_workspace_bytes(T))
        return EMBER_ERR_WORKSPACE;
    const cudaStream_t s = (cudaStream_t)stream;
    LossArgs a{};
    a.z = logits;
    a.y = targets;
    a.w = weights;
    a.d = dlogits;
    a.nll = nll;
    a.loss = loss;
    a.total = static_cast<double *>(workspace);
    a.count = reinterpret_cast<int *>(a.total + kMaxParts);
    a.status = status;
    a.ticket = status + 1;
    a.wait_ns = ops_wait_ns();
    a.ldz = ldz;
    a.ldd = ldd;
    a.T = T;
    a.V = V;
    a.ignore = ignore_index;
    a.y64 = idtype == EMBER_I64;
    a.mean = mean;
    if (T == 0)
        return launched(cudaMemsetAsync(loss, 0, sizeof(float), s));
    const bool zb = ztype == EMBER_BF16, db = dtype == EMBER_BF16;
    cudaError_t e;
    if (!dlogits)
        e = zb ? launch_rows<bf16_t, bf16_t, false>(a, s) : launch_rows<float, float, false>(a, s);
    else if (zb)
        e = db ? launch_rows<bf16_t, bf16_t, true>(a, s) : launch_rows<bf16_t, float, true>(a, s);
    else
        e = db ? launch_rows<float, bf16_t, true>(a, s) : launch_rows<float, float, true>(a, s);
    return launched(e);
}

// The status block of the operators that report what only the GPU sees: the
// sticky flags and a counter that each call leaves at zero.
ember_status ember_status_init(unsigned *status, void *stream)
{
    if (!status)
        return EMBER_ERR_INVALID_ARG;
    if (!aligned(status, 4))
        return EMBER_ERR_ALIGNMENT;
    return launched(cudaMemsetAsync(status, 0, EMBER_STATUS_BYTES, (cudaStream_t)stream));
}

ember_status ember_set_ops_wait_limit(uint64_t ns)
{
    ops_wait.store(ns ? ns : kDefaultWaitNs, std::memory_order_relaxed);
    return EMBER_OK;
}

ember_status ember_status_read(unsigned *status, void *stream)
{
    if (!status)
        return EMBER_ERR_INVALID_ARG;
    if (!aligned(status, 4))
        return EMBER_ERR_ALIGNMENT;
    const cudaStream_t s = (cudaStream_t)stream;
    unsigned flags = 0;
    cudaError_t e = cudaMemcpyAsync(&flags, status, sizeof(flags), cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess)
        e = cudaStreamSynchronize(s);
    if (e == cudaSuccess && flags)
        e = cudaMemsetAsync(status, 0, sizeof(flags), s);
    if (e != cudaSuccess)
        return launched(e);
    return (flags & kFlagTimeout) ? EMBER_ERR_TIMEOUT : (flags & kFlagIdRange) ? EMBER_ERR_ID_OUT_OF_RANGE : EMBER_OK;
}

}  // extern "C"
