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
// A row of up to 262144 logits is spread over a cluster of up to 8 CTAs and
// stays in their registers between the statistics and the gradient; the CTAs
// exchange one pair each through distributed shared memory.
#include "ember_rows.cuh"
#include "ember_tc.cuh"

namespace ember {
namespace {

using namespace rows;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_huge_valf();

// 2^x, and e^x of a difference: the difference is exact where it matters
// (near zero), so its rounding costs a relative 2^-23 |x| at most.
__device__ __forceinline__ float exp_of(float d) { return exp2f(d * kLog2e); }

struct MaxSum {
    float m, s;
};
// A maximum of -inf (nothing seen but -inf) is replaced by 0 in differences,
// so that exp gives 0 and not NaN.
__device__ __forceinline__ float finite_max(float m) { return m == -kInf ? 0.f : m; }
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b)
{
    MaxSum r;
    r.m = fmaxf(a.m, b.m);
    const float m = finite_max(r.m);
    r.s = a.s * exp_of(a.m - m) + b.s * exp_of(b.m - m);
    return r;
}
__device__ __forceinline__ MaxSum warp_join(MaxSum v)
{
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1)
        v = join(v, {__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o)});
    return v;
}

struct LossArgs {
    const void *z, *y;
    const float *w;
    void *d;
    float *nll, *loss;
    long long *count;
    unsigned *status;
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

// The number of counted tokens, by one CTA.
__global__ void __launch_bounds__(1024) k_loss_count(LossArgs a)
{
    __shared__ long long part[32];
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    long long n = 0;
    bool bad = false;
    for (int64_t t = threadIdx.x; t < a.T; t += blockDim.x) {
        const int64_t y = target_of(a, t);
        n += counts(a, y);
        bad |= y != a.ignore && !counts(a, y);
    }
    if (bad)
        atomicOr(a.status, kFlagIdRange);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1)
        n += __shfl_xor_sync(0xffffffffu, n, o);
    if ((threadIdx.x & 31) == 0)
        part[threadIdx.x >> 5] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
        n = 0;
        for (int k = 0; k < 32; ++k)
            n += part[k];
        *a.count = n;
    }
}

// The total, by one CTA: each thread adds its tokens in order, then a tree.
__global__ void __launch_bounds__(1024) k_loss_total(LossArgs a)
{
    __shared__ double part[32];
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    double s = 0.0;
    for (int64_t t = threadIdx.x; t < a.T; t += blockDim.x)
        if (counts(a, target_of(a, t)))
            s += (double)a.nll[t] * (a.w ? (double)a.w[t] : 1.0);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1)
        s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0)
        part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int k = 0; k < 32; ++k)
            s += part[k];
        const long long n = a.mean ? *a.count : 1;
        *a.loss = n > 0 ? (float)(s / (double)n) : 0.f;
    }
}

__device__ __forceinline__ float row_gain(const LossArgs &a, int64_t t)
{
    const float w = a.w ? a.w[t] : 1.f;
    return a.mean ? w / (float)*a.count : w;
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
    ms = warp_join(ms);
    if ((threadIdx.x & 31) == 0)
        part[threadIdx.x >> 5] = ms;
    __syncthreads();
    ms = warp_join(part[threadIdx.x & 31]);
    const float m = finite_max(ms.m);
    if (threadIdx.x == 0)
        a.nll[t] = ms.s == 0.f ? kInf : m - zy[0] + logf(ms.s);
    if (!GRAD)
        return;
    const float g = row_gain(a, t);
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

// One cluster per row.  The row is cut at the 16-byte groups (32-byte for
// fp32) of its address into groups of 8 logits, NG per thread; the up to 14
// logits before the first and after the last whole group go one by one to
// threads of the first CTA.  The gradient's rows are at the same places of
// their groups (launch_rows sees to it).
template <typename ZT, typename DT, bool GRAD, int NG, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) k_loss_cluster(LossArgs a, int count_here)
{
    __shared__ MaxSum part[32];
    __shared__ MaxSum all[8];
    __shared__ int nvalid[32];
    const unsigned C = tc::cluster_count_in(), rank = tc::cluster_rank();
    const int64_t t = blockIdx.x / C;
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5, nwarps = nt >> 5;
    if (C > 1)
        tc::cluster_arrive();  // waited for before the first store into another CTA: by then all have started
    dev::grid_dep_wait();
    dev::grid_dep_launch();

    const int64_t y = target_of(a, t);
    const bool on = counts(a, y);
    const ZT *z = static_cast<const ZT *>(a.z) + t * a.ldz;
    DT *d = static_cast<DT *>(a.d) + t * a.ldd;
    const int V = (int)a.V;
    int head = (int)((8 - ((uintptr_t)z / sizeof(ZT)) % 8) % 8);
    head = head < V ? head : V;
    const int ngroups = (V - head) / 8;
    const int tail = V - head - ngroups * 8;
    const int first = (int)rank * nt + tid, step = (int)C * nt;
    // the logit outside the groups that this thread has, or -1
    int single = -1;
    if (rank == 0 && tid < head + tail)
        single = tid < head ? tid : V - tail + (tid - head);

    Raw<ZT, 8> r[NG];
    float zs = -kInf;
    if (on) {
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            const int g = first + k * step;
            if (g < ngroups)
                r[k] = load_raw<ZT, 8>(z + head + (int64_t)g * 8);
        }
        if (single >= 0) {
            float f[1];
            unpack<ZT, 1>(load_raw<ZT, 1>(z + single), f);
            zs = f[0];
        }
    }
    float zy[1] = {0.f};
    if (on && rank == 0 && tid == 0)
        unpack<ZT, 1>(load_raw<ZT, 1>(z + y), zy);
    // the number of counted tokens: from the kernel before, or, when the
    // tokens are few, from their targets at once
    float n = 1.f;
    if (count_here) {
        int c = 0;
        bool bad = false;
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
    } else if (a.mean)
        n = (float)*a.count;

    MaxSum ms{zs, 0.f};
#pragma unroll
    for (int k = 0; k < NG; ++k)
        if (on && first + k * step < ngroups) {
            float f[8];
            unpack<ZT, 8>(r[k], f);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                ms.m = fmaxf(ms.m, f[e]);
        }
    {
        const float m = finite_max(ms.m);
        ms.s = exp_of(zs - m);
#pragma unroll
        for (int k = 0; k < NG; ++k)
            if (on && first + k * step < ngroups) {
                float f[8];
                unpack<ZT, 8>(r[k], f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    ms.s += exp_of(f[e] - m);
            }
    }
    ms = warp_join(ms);
    if (lane == 0)
        part[warp] = ms;
    __syncthreads();
    ms = warp_join(lane < nwarps ? part[lane] : MaxSum{-kInf, 0.f});
    if (C > 1) {
        // every CTA's pair into every CTA
        tc::cluster_wait();
        if (tid < (int)C)
            tc::store_remote(&all[rank], tid, ms.m, ms.s);
        tc::cluster_sync();
        ms = all[0];
        for (unsigned k = 1; k < C; ++k)
            ms = join(ms, all[k]);
    }
    if (count_here) {
        int c = 0;
        for (int k = 0; k < nwarps; ++k)
            c += nvalid[k];
        n = (float)c;
        if (blockIdx.x == 0 && tid == 0)
            *a.count = c;
    }
    const float m = finite_max(ms.m);
    if (rank == 0 && tid == 0)
        a.nll[t] = !on ? 0.f : ms.s == 0.f ? kInf : m - zy[0] + logf(ms.s);
    if constexpr (GRAD) {
        float g = on ? (a.w ? a.w[t] : 1.f) : 0.f;
        if (a.mean && on)
            g /= n;
        const bool live = on && ms.s != 0.f;
        const float f = live ? g / ms.s : 0.f;
        const float hot = live ? g : 0.f;
        const int yg = on ? ((int)y - head) : -1;  // place of the target among the groups' logits
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            const int gi = first + k * step;
            if (gi < ngroups) {
                float o[8];
                if (live) {
                    unpack<ZT, 8>(r[k], o);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        o[e] = exp_of(o[e] - m) * f;
                    if (yg >= 0 && (yg >> 3) == gi) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if ((yg & 7) == e)
                                o[e] -= hot;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        o[e] = 0.f;
                }
                store_group<DT, 8>(d + head + (int64_t)gi * 8, o);
            }
        }
        if (single >= 0) {
            const float o[1] = {live ? exp_of(zs - m) * f - (single == (int)y ? hot : 0.f) : 0.f};
            store_group<DT, 1>(d + single, o);
        }
    }
}

// Threads per CTA and CTAs per row for rows of V logits, or C = 0 where the
// row does not fit the registers of a cluster.  Four groups a thread (16 KiB
// of bf16 logits per 256 threads in flight); CTAs of up to 512 threads, so
// that several rows share an SM and one row's loads cover another's stores.
struct RowPlan {
    int C, nt;
};
constexpr int kLossGroups = 4;
constexpr int64_t kCountHere = 512;  // tokens whose targets every CTA counts itself

RowPlan row_plan(int64_t T, int64_t V)
{
    RowPlan p{0, 0};
    const int64_t threads = (V / 8 + kLossGroups - 1) / kLossGroups;
    int C = 1;
    while (C < 8 && threads > (int64_t)C * 512)
        C *= 2;
    if (threads > (int64_t)C * 1024 || T * C > INT32_MAX)
        return p;
    p.C = C;
    p.nt = (int)((threads + C - 1) / C + 31) / 32 * 32;
    if (p.nt < 32)
        p.nt = 32;
    return p;
}

template <typename ZT, typename DT, bool GRAD>
cudaError_t launch_rows(const LossArgs &a, cudaStream_t stream)
{
    RowPlan p = row_plan(a.T, a.V);
    if (GRAD && (((uintptr_t)a.z / sizeof(ZT) - (uintptr_t)a.d / sizeof(DT)) % 8 != 0 || (a.ldz - a.ldd) % 8 != 0))
        p.C = 0;
    const bool here = p.C > 0 && a.T <= kCountHere;
    cudaError_t e = cudaSuccess;
    if (!here)
        e = launch_k(k_loss_count, dim3(1), dim3(1024), 0, stream, true, a);
    if (e != cudaSuccess)
        return e;
    if (p.C == 0)
        return launch_k(k_loss_stream<ZT, DT, GRAD>, dim3((unsigned)a.T), dim3(1024), 0, stream, true, a);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.T * p.C));
    cfg.blockDim = dim3(p.nt);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = p.C;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (p.nt <= 512)
        return cudaLaunchKernelEx(&cfg, k_loss_cluster<ZT, DT, GRAD, kLossGroups, 512, sizeof(ZT) == 2 ? 3 : 2>, a,
                                  (int)here);
    return cudaLaunchKernelEx(&cfg, k_loss_cluster<ZT, DT, GRAD, kLossGroups, 1024, 1>, a, (int)here);
}

}  // namespace
}  // namespace ember

using namespace ember;

extern "C" {

size_t ember_softmax_loss_workspace_bytes(int64_t T)
{
    return T >= 0 && T <= INT32_MAX ? 256 : 0;
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
    a.count = static_cast<long long *>(workspace);
    a.status = status;
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
    if (e == cudaSuccess)
        e = launch_k(k_loss_total, dim3(1), dim3(1024), 0, s, true, a);
    return launched(e);
}

// The sticky word of the operators that report what only the GPU sees.
ember_status ember_status_init(unsigned *status, void *stream)
{
    if (!status)
        return EMBER_ERR_INVALID_ARG;
    if (!aligned(status, 4))
        return EMBER_ERR_ALIGNMENT;
    return launched(cudaMemsetAsync(status, 0, sizeof(unsigned), (cudaStream_t)stream));
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
