// Matrix product in 8-bit integers with a scale per token and per channel:
//
//   out[t][v] = xs[t] ws[v] sum_k xq[t][k] wq[v][k]
//
// the logits of a head whose table is kept in 8 bits (ember_quantize_rows)
// and whose hidden states the norm wrote in 8 bits (ember_rmsnorm_quant).
#include "ember_rows.cuh"

namespace ember {
namespace {

using namespace rows;

struct MmArgs {
    const int8_t *xq, *wq;
    const float *xs, *ws;
    void *out;
    int64_t ldx, ldw, ldo, T, V;
    int K;
};

__device__ __forceinline__ void store_out(void *out, int obf16, int64_t at, float v)
{
    if (obf16)
        static_cast<unsigned short *>(out)[at] = dev::f2bf(v);
    else
        static_cast<float *>(out)[at] = v;
}

// Rows at any address: tiles of 64 channels x 16 tokens through shared
// memory, loaded byte by byte, the products by four with dp4a.  Takes what
// the kernels with 16-byte loads cannot.
constexpr int kGV = 64, kGT = 16, kGK = 64;
__global__ void __launch_bounds__(256) k_mm_any(MmArgs a, int obf16, unsigned vblocks)
{
    __shared__ int sx[kGT][kGK / 4 + 1];
    __shared__ int sw[kGV][kGK / 4 + 1];
    const int64_t v0 = (int64_t)(blockIdx.x % vblocks) * kGV, t0 = (int64_t)(blockIdx.x / vblocks) * kGT;
    const int tv = threadIdx.x & 63, tt = threadIdx.x >> 6;
    int acc[4] = {0, 0, 0, 0};
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    for (int k0 = 0; k0 < a.K; k0 += kGK) {
        for (int i = threadIdx.x; i < (kGT + kGV) * kGK; i += 256) {
            const int r = i / kGK, k = i % kGK;
            int8_t q = 0;
            if (k0 + k < a.K) {
                if (r < kGT) {
                    if (t0 + r < a.T)
                        q = a.xq[(t0 + r) * a.ldx + k0 + k];
                } else if (v0 + r - kGT < a.V)
                    q = a.wq[(v0 + r - kGT) * a.ldw + k0 + k];
            }
            if (r < kGT)
                reinterpret_cast<int8_t *>(sx[r])[k] = q;
            else
                reinterpret_cast<int8_t *>(sw[r - kGT])[k] = q;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kGK / 4; ++k) {
            const int w = sw[tv][k];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[j] = __dp4a(sx[tt + 4 * j][k], w, acc[j]);
        }
        __syncthreads();
    }
    const int64_t v = v0 + tv;
    if (v >= a.V)
        return;
    const float ws = a.ws[v];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t t = t0 + tt + 4 * j;
        if (t < a.T)
            store_out(a.out, obf16, t * a.ldo + v, (float)acc[j] * a.xs[t] * ws);
    }
}

}  // namespace
}  // namespace ember

using namespace ember;

extern "C" {

size_t ember_matmul_quant_workspace_bytes(int64_t T, int64_t V, int64_t K)
{
    if (T < 0 || V < 1 || K < 1 || T > INT32_MAX || V > INT32_MAX || K > kMaxRowCols)
        return 0;
    return 256;
}

ember_status ember_matmul_quant(const int8_t *xq, int64_t ldx, const float *xs, const int8_t *wq, int64_t ldw,
                                const float *ws, int64_t T, int64_t V, int64_t K, void *out, int64_t ldo,
                                ember_wdtype otype, void *workspace, size_t bytes, unsigned *status, void *stream)
{
    if (T < 0 || V < 1 || K < 1 || ldx < K || ldw < K || ldo < V || !wq || !ws || !status)
        return EMBER_ERR_INVALID_ARG;
    if (T > 0 && (!xq || !xs || !out))
        return EMBER_ERR_INVALID_ARG;
    if (!dtype_ok(otype))
        return EMBER_ERR_DTYPE;
    if (T > INT32_MAX || V > INT32_MAX || K > kMaxRowCols || ldx > (int64_t(1) << 31) || ldw > (int64_t(1) << 31) ||
        ldo > (int64_t(1) << 32))
        return EMBER_ERR_UNSUPPORTED;
    if (!aligned(xs, 4) || !aligned(ws, 4) || !aligned(out, elem_size(otype)) || !aligned(status, 4) ||
        !aligned(workspace, 16))
        return EMBER_ERR_ALIGNMENT;
    if (T == 0)
        return EMBER_OK;
    if (!workspace || bytes < ember_matmul_quant_workspace_bytes(T, V, K))
        return EMBER_ERR_WORKSPACE;
    MmArgs a{xq, wq, xs, ws, out, ldx, ldw, ldo, T, V, (int)K};
    const int64_t vb = (V + kGV - 1) / kGV, tb = (T + kGT - 1) / kGT;
    if (vb * tb > INT32_MAX)
        return EMBER_ERR_UNSUPPORTED;
    return launched(launch_k(k_mm_any, dim3((unsigned)(vb * tb)), dim3(256), 0, (cudaStream_t)stream, true, a,
                             (int)(otype == EMBER_BF16), (unsigned)vb));
}

}  // extern "C"
