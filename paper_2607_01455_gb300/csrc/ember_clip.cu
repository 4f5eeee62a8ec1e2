// The global norm over many gradients and their clipping:
//
//   norm = sqrt(sum over all tensors of g^2)
//   out = g min(1, max_norm / (norm + eps))
//
// Both passes are bound by HBM (L2 for small sets).  All tensors of a call go
// into one launch: their addresses, sizes and types travel as kernel
// arguments (up to kManyTensors of them; more take more launches), and the
// elements are cut into chunks that CTAs take in turn, whatever tensor they
// belong to.  The norm pass leaves one 64-bit sum per CTA; every CTA of the
// scaling pass adds them itself, in order, so nothing waits for a last CTA.
//
// A thread adds the squares of its 8 or 32 values of a chunk in 32 bits and
// carries the sums of chunks in 64 (GB300 adds about two 64-bit values per
// clock and SM, so one per 8 values would set the pace); where the squares leave the range of 32
// bits (values above 1e15 or below 1e-13) that thread's values are squared in
// 64 bits instead, so the norm neither overflows nor loses small gradients.
//
// Measured: 200 M fp32 gradients, norm 117 us (6.8 TB/s, DRAM 87 % busy), scaling
// 247 us (6.5 TB/s); a set above L2 is read twice, so clipping 400 M mixed ones
// takes 0.50 ms against 0.31 ms for reading and writing them once.
#include "ember_rows.cuh"

namespace ember {
namespace {

using namespace rows;

constexpr int kClipThreads = 512;
constexpr int kClipCtas = kSms * 2;
// Tensors of a launch: the host copies the whole list for each (clipping 100
// tensors of 1000 with 256 places 8.8 us, with 1024 10.7).
constexpr int kFewTensors = 64, kSomeTensors = 256, kManyTensors = 1024;

template <int CAP>
struct TensorList {
    const void *in[CAP];
    void *out[CAP];
    int64_t n[CAP];            // elements, with kBf16Bit set for bf16
    unsigned start[CAP + 1];   // first chunk of each tensor
    int count;
};
constexpr int64_t kBf16Bit = int64_t(1) << 62;
static_assert(sizeof(TensorList<kManyTensors>) < 32000, "kernel arguments end at 32764 bytes");

struct ClipArgs {
    double *part;     // one sum per CTA of the norm pass
    int nparts;
    float *norm;      // written by the first CTA of the scaling pass
    float max_norm, eps;
    int in_place;
};

// Tensor of chunk c: the last one that starts at or before it.
template <int CAP>
__device__ __forceinline__ int tensor_of(const TensorList<CAP> &l, unsigned c)
{
    int lo = 0, hi = l.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (l.start[mid] <= c)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// Sum of squares of N values: in 32 bits, in four chains, or nothing and
// `wide` set where it must be done in 64.  A sum of zero is among those: zeros
// and values whose squares vanish look alike in it, so groups of nothing but
// zeros are read a second time too (right, but slower than others).
template <int N>
__device__ __forceinline__ double squares(const float (&v)[N], bool &wide)
{
    float p[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < N; ++e)
        p[e & 3] = fmaf(v[e], v[e], p[e & 3]);
    const float s = (p[0] + p[1]) + (p[2] + p[3]);
    wide = !(s >= 1e-25f && s <= 1e30f);
    return wide ? 0.0 : (double)s;
}

// Elements of a tensor before its first 16-byte (bf16) or 32-byte (fp32)
// group; they are taken one by one by its first chunk, and what is left
// behind the last whole group by its last one.
template <typename T>
__device__ __forceinline__ int head_of(const T *p, int64_t n)
{
    const int h = (int)((8 - ((uintptr_t)p / sizeof(T)) % 8) % 8);
    return h < n ? h : (int)n;
}

// This thread's groups of a chunk.  A chunk that lies inside the tensor loads
// without a test between the loads, so that all of them are in flight.
template <typename T, int NG>
__device__ __forceinline__ void load_chunk(const T *body, int64_t g0, int64_t ngroups, Raw<T, 8> (&r)[NG])
{
    if (g0 + NG * kClipThreads <= ngroups) {
        const T *p = body + (g0 + threadIdx.x) * 8;
#pragma unroll
        for (int k = 0; k < NG; ++k)
            r[k] = load_raw<T, 8>(p + k * (kClipThreads * 8));
    } else {
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            const int64_t g = g0 + k * kClipThreads + threadIdx.x;
            r[k] = g < ngroups ? load_raw<T, 8>(body + g * 8) : zero_raw<T, 8>();
        }
    }
}

template <typename T, int NG>
__device__ __forceinline__ double chunk_squares(const T *p, int64_t n, unsigned chunk)
{
    const int head = head_of(p, n);
    const int64_t ngroups = (n - head) / 8;
    const int64_t g0 = (int64_t)chunk * (NG * kClipThreads);
    const T *body = p + head;
    Raw<T, 8> r[NG];
    load_chunk<T, NG>(body, g0, ngroups, r);
    float v[NG * 8];
#pragma unroll
    for (int k = 0; k < NG; ++k) {
        float f[8];
        unpack<T, 8>(r[k], f);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[k * 8 + e] = f[e];
    }
    bool wide;
    double s = squares<NG * 8>(v, wide);
    if (wide)  // read again, so that the values need not be kept for it
        for (int k = 0; k < NG; ++k) {
            const int64_t g = g0 + k * kClipThreads + threadIdx.x;
            for (int e = 0; g < ngroups && e < 8; ++e) {
                float f[1];
                unpack<T, 1>(load_raw<T, 1>(body + g * 8 + e), f);
                if (f[0] != 0.f)
                    s += (double)f[0] * (double)f[0];
            }
        }
    if (chunk == 0) {  // the elements outside whole groups, at most 14
        const int tail = (int)(n - head - ngroups * 8);
        if ((int)threadIdx.x < head + tail) {
            const int64_t at = (int)threadIdx.x < head ? threadIdx.x : n - tail + ((int)threadIdx.x - head);
            float f[1];
            unpack<T, 1>(load_raw<T, 1>(p + at), f);
            s += (double)f[0] * (double)f[0];
        }
    }
    return s;
}

// The sum over the CTA, in the first warp, in a fixed order.  The SM adds two
// 64-bit values a clock, 16 clocks per warp: the other warps would only queue
// before the one that counts (clipping 12 tensors of 8000, with the root in one
// warp too: 8.0 us to 4.5, 40 of 50000: 14.7 to 6.4).
__device__ __forceinline__ double block_sum(double s)
{
    __shared__ double part[kClipThreads];
    part[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        double c[4];
#pragma unroll
        for (int k = 0; k < kClipThreads / 32; ++k) {
            const double v = part[k * 32 + threadIdx.x];
            c[k & 3] = k < 4 ? v : c[k & 3] + v;
        }
        s = (c[0] + c[1]) + (c[2] + c[3]);
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1)
            s += __shfl_xor_sync(0xffffffffu, s, o);
    }
    return s;
}

template <int CAP, int NG>
__global__ void __launch_bounds__(kClipThreads) k_norm_parts(const __grid_constant__ TensorList<CAP> l, double *part)
{
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    double s = 0.0;
    const unsigned nchunks = l.start[l.count];
    for (unsigned c = blockIdx.x; c < nchunks; c += gridDim.x) {
        const int i = tensor_of(l, c);
        const int64_t n = l.n[i] & (kBf16Bit - 1);
        const unsigned chunk = c - l.start[i];
        if (l.n[i] & kBf16Bit)
            s += chunk_squares<bf16_t, NG>(static_cast<const bf16_t *>(l.in[i]), n, chunk);
        else
            s += chunk_squares<float, NG>(static_cast<const float *>(l.in[i]), n, chunk);
    }
    s = block_sum(s);
    if (threadIdx.x == 0)
        part[blockIdx.x] = s;
}

// The norm from the parts, the same bits in every CTA.
__device__ __forceinline__ float norm_of(const double *part, int nparts)
{
    __shared__ float norm;
    double s = (int)threadIdx.x < nparts ? __ldcg(part + threadIdx.x) : 0.0;
    for (int k = threadIdx.x + kClipThreads; k < nparts; k += kClipThreads)
        s += __ldcg(part + k);
    s = block_sum(s);
    if (threadIdx.x < 32) {
        const float n = (float)sqrt(s);
        if (threadIdx.x == 0)
            norm = n;
    }
    __syncthreads();
    return norm;
}

__global__ void __launch_bounds__(kClipThreads) k_norm_total(const double *part, int nparts, float *norm)
{
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    const float n = norm_of(part, nparts);
    if (threadIdx.x == 0)
        *norm = n;
}

template <typename T, int NG>
__device__ __forceinline__ void chunk_scale(const T *p, T *o, int64_t n, unsigned chunk, float c)
{
    const int head = head_of(p, n);
    const int64_t ngroups = (n - head) / 8;
    const int64_t g0 = (int64_t)chunk * (NG * kClipThreads);
    const T *body = p + head;
    Raw<T, 8> r[NG];
    load_chunk<T, NG>(body, g0, ngroups, r);
    const bool whole = (uintptr_t)(o + head) % (8 * sizeof(T)) == 0;
#pragma unroll
    for (int k = 0; k < NG; ++k) {
        const int64_t g = g0 + k * kClipThreads + threadIdx.x;
        if (g < ngroups) {
            float f[8];
            unpack<T, 8>(r[k], f);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                f[e] *= c;
            T *to = o + head + g * 8;
            if (whole)
                store_group<T, 8>(to, f);
            else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float one[1] = {f[e]};
                    store_group<T, 1>(to + e, one);
                }
            }
        }
    }
    if (chunk == 0) {
        const int tail = (int)(n - head - ngroups * 8);
        if ((int)threadIdx.x < head + tail) {
            const int64_t at = (int)threadIdx.x < head ? threadIdx.x : n - tail + ((int)threadIdx.x - head);
            float f[1];
            unpack<T, 1>(load_raw<T, 1>(p + at), f);
            f[0] *= c;
            store_group<T, 1>(o + at, f);
        }
    }
}

template <int CAP, int NG>
__global__ void __launch_bounds__(kClipThreads) k_clip_scale(const __grid_constant__ TensorList<CAP> l, ClipArgs a)
{
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    const float norm = norm_of(a.part, a.nparts);
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *a.norm = norm;
    float c = a.max_norm / (norm + a.eps);
    c = c > 1.f ? 1.f : c;  // a NaN stays one
    if (c == 1.f && a.in_place)
        return;  // nothing changes
    const unsigned nchunks = l.start[l.count];
    // the last chunks first: the norm pass has left them in L2
    for (unsigned k = blockIdx.x; k < nchunks; k += gridDim.x) {
        const unsigned ch = nchunks - 1 - k;
        const int i = tensor_of(l, ch);
        const int64_t n = l.n[i] & (kBf16Bit - 1);
        const unsigned chunk = ch - l.start[i];
        if (l.n[i] & kBf16Bit)
            chunk_scale<bf16_t, NG>(static_cast<const bf16_t *>(l.in[i]), static_cast<bf16_t *>(l.out[i]), n, chunk, c);
        else
            chunk_scale<float, NG>(static_cast<const float *>(l.in[i]), static_cast<float *>(l.out[i]), n, chunk, c);
    }
}

// Chunks of 8 elements per thread while the whole set has fewer chunks than
// four per CTA, of 32 otherwise.
constexpr int64_t kSmallChunk = 8 * kClipThreads, kLargeChunk = 32 * kClipThreads;

constexpr int64_t kMaxTotal = int64_t(1) << 42;  // elements of a call: 8 TiB of bf16

struct Tensors {
    const void *const *in;
    void *const *out;
    const int64_t *numel;
    const int *types;
    int n;
};

template <int CAP>
int fill(TensorList<CAP> &l, const Tensors &t, int first, int64_t chunk)
{
    l.count = 0;
    l.start[0] = 0;
    int k = first;
    for (; k < t.n && l.count < CAP; ++k) {
        if (t.numel[k] == 0)
            continue;
        const int64_t chunks = (t.numel[k] + chunk - 1) / chunk;  // below 2^29 in all, see kMaxTotal
        l.in[l.count] = t.in[k];
        l.out[l.count] = t.out ? t.out[k] : nullptr;
        l.n[l.count] = t.numel[k] | (t.types[k] == EMBER_BF16 ? kBf16Bit : 0);
        l.start[l.count + 1] = l.start[l.count] + (unsigned)chunks;
        ++l.count;
    }
    return k;
}

template <int CAP, int NG>
cudaError_t passes(const Tensors &t, int64_t chunk, bool scale, ClipArgs a, cudaStream_t stream)
{
    TensorList<CAP> l;
    a.nparts = 0;
    for (int k = 0; k < t.n;) {
        k = fill(l, t, k, chunk);
        if (l.count == 0)
            continue;
        const unsigned n = l.start[l.count];
        const int grid = n < kClipCtas ? (int)n : kClipCtas;
        const cudaError_t e = launch_k(k_norm_parts<CAP, NG>, dim3(grid), dim3(kClipThreads), 0, stream, true, l,
                                       a.part + a.nparts);
        if (e != cudaSuccess)
            return e;
        a.nparts += grid;
    }
    if (!scale || a.nparts == 0)
        return launch_k(k_norm_total, dim3(1), dim3(kClipThreads), 0, stream, true, (const double *)a.part, a.nparts,
                        a.norm);
    for (int k = 0; k < t.n;) {
        k = fill(l, t, k, chunk);
        if (l.count == 0)
            continue;
        const unsigned n = l.start[l.count];
        const cudaError_t e = launch_k(k_clip_scale<CAP, NG>, dim3(n < kClipCtas ? n : kClipCtas), dim3(kClipThreads), 0,
                                       stream, true, l, a);
        if (e != cudaSuccess)
            return e;
    }
    return cudaSuccess;
}

ember_status check(const Tensors &t, void *workspace, size_t bytes, float *norm)
{
    if (t.n < 0 || !norm || (t.n > 0 && (!t.in || !t.numel || !t.types)))
        return EMBER_ERR_INVALID_ARG;
    int64_t total = 0;
    for (int k = 0; k < t.n; ++k) {
        if (t.numel[k] < 0 || (t.numel[k] > 0 && (!t.in[k] || (t.out && !t.out[k]))))
            return EMBER_ERR_INVALID_ARG;
        if (!dtype_ok(t.types[k]))
            return EMBER_ERR_DTYPE;
        if (t.numel[k] > 0 && (!aligned(t.in[k], elem_size(t.types[k])) ||
                               (t.out && !aligned(t.out[k], elem_size(t.types[k])))))
            return EMBER_ERR_ALIGNMENT;
        if (t.numel[k] > kMaxTotal || (total += t.numel[k]) > kMaxTotal)
            return EMBER_ERR_UNSUPPORTED;
    }
    if (!aligned(norm, 4) || !aligned(workspace, 16))
        return EMBER_ERR_ALIGNMENT;
    if (!workspace || bytes < ember_clip_workspace_bytes(t.n))
        return EMBER_ERR_WORKSPACE;
    return EMBER_OK;
}

cudaError_t run(const Tensors &t, bool scale, const ClipArgs &a, cudaStream_t stream)
{
    int64_t total = 0;
    for (int k = 0; k < t.n; ++k)
        total += t.numel[k];
    const bool brief = total < 4 * kClipCtas * kSmallChunk;
    if (t.n <= kFewTensors)
        return brief ? passes<kFewTensors, 1>(t, kSmallChunk, scale, a, stream)
                     : passes<kFewTensors, 4>(t, kLargeChunk, scale, a, stream);
    if (t.n <= kSomeTensors)
        return brief ? passes<kSomeTensors, 1>(t, kSmallChunk, scale, a, stream)
                     : passes<kSomeTensors, 4>(t, kLargeChunk, scale, a, stream);
    return brief ? passes<kManyTensors, 1>(t, kSmallChunk, scale, a, stream)
                 : passes<kManyTensors, 4>(t, kLargeChunk, scale, a, stream);
}

}  // namespace
}  // namespace ember

using namespace ember;

extern "C" {

size_t ember_clip_workspace_bytes(int n)
{
    if (n < 0)
        return 0;
    // one sum per CTA of each launch of up to kManyTensors tensors
    return sizeof(double) * (size_t)kClipCtas * (size_t)(n / kManyTensors + 1);
}

ember_status ember_grad_norm(int n, const void *const *grads, const int64_t *numel, const int *types, float *norm,
                             void *workspace, size_t bytes, void *stream)
{
    const Tensors t{grads, nullptr, numel, types, n};
    const ember_status st = check(t, workspace, bytes, norm);
    if (st != EMBER_OK)
        return st;
    ClipArgs a{};
    a.part = static_cast<double *>(workspace);
    a.norm = norm;
    return launched(run(t, false, a, (cudaStream_t)stream));
}

ember_status ember_clip_grads(int n, const void *const *grads, void *const *out, const int64_t *numel,
                              const int *types, float max_norm, float eps, float *norm, void *workspace, size_t bytes,
                              void *stream)
{
    if (!(max_norm >= 0.f) || !(eps >= 0.f) || (n > 0 && !out))
        return EMBER_ERR_INVALID_ARG;
    const Tensors t{grads, out, numel, types, n};
    const ember_status st = check(t, workspace, bytes, norm);
    if (st != EMBER_OK)
        return st;
    ClipArgs a{};
    a.part = static_cast<double *>(workspace);
    a.norm = norm;
    a.max_norm = max_norm;
    a.eps = eps;
    a.in_place = 1;
    for (int k = 0; k < n; ++k)
        if (numel[k] > 0 && grads[k] != out[k])
            a.in_place = 0;
    return launched(run(t, true, a, (cudaStream_t)stream));
}

}  // extern "C"
