// Matrix product in 8-bit integers with a scale per token and per channel:
//
//   out[t][v] = xs[t] ws[v] sum_k xq[t][k] wq[v][k]
//
// the logits of a head whose table is kept in 8 bits (ember_quantize_rows)
// and whose hidden states the norm wrote in 8 bits (ember_rmsnorm_quant).
//
// Three kernels, by the number of tokens and the rows' alignment:
//   k_mm_few   up to 4 tokens, up to 8 by all but large tables, more by a small
//              table of short rows in groups of 8 while all groups run at once:
//              each group reads the table once, the products by dp4a; bound by HBM.
//   k_mm_tc    more tokens: tcgen05 on pairs of CTAs; bound by HBM up to
//              about 128 tokens, by the tensor cores beyond.
//   k_mm_any   tables whose rows do not start on 16 bytes.
//
// GB300's tensor cores have no fast 8-bit integer form, but an 8-bit integer
// is an fp16 number: k_mm_tc widens the table's tiles on their way into
// tensor memory and multiplies in fp16 with fp32 sums.  Products of two
// 8-bit integers and sums of them below 2^24 are exact in fp32, so the result
// is the integer one as long as sum_k |xq wq| < 2^24 (always for K <= 1024,
// and for hidden states and tables in use far beyond); past that the tensor
// cores cut the sum off after each step of 16 products, at most two ulps a step.
// The other two kernels sum 32-bit integers: beyond 2^24 the bits depend on
// which kernel a call takes, and so on T.
#include "ember_rows.cuh"
#include "ember_tc.cuh"

#include <cuda_fp16.h>

namespace ember {
namespace {

using namespace rows;

constexpr int64_t kMaxMmRows = INT32_MAX - 1024;  // row numbers of a last tile stay within 32 bits

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


// ---------------------------------------------------------------------------
// Few tokens, a row of the grid per group of TN.  The tokens' rows sit in shared
// memory, zero-padded to whole 512-byte slabs; a warp takes R rows of the table
// at a time, 16 bytes of each row per lane and slab, so that every 16 bytes of x
// are read from shared memory once for R rows.  The lanes' integer sums are
// joined by a transposed butterfly: R TN totals for about as many shuffles.
// Bound by HBM for one to four tokens: 128256 x 8192 for one token 145 us, 7.2
// TB/s; for eight, dp4a sets the pace (195 us).
// ---------------------------------------------------------------------------
constexpr int kFewTokens = 8;
constexpr int kFewThreads = 256;
constexpr size_t kFewSmem = 100 << 10;  // two CTAs per SM

template <int R>
__device__ __forceinline__ int warp_isum_transposed(int (&v)[R], int lane, int &index)
{
    constexpr int kLog = R >= 32 ? 5 : R >= 16 ? 4 : R >= 8 ? 3 : R >= 4 ? 2 : R >= 2 ? 1 : 0;
    static_assert((1 << kLog) == R, "a power of two up to 32");
    index = 0;
#pragma unroll
    for (int s = 0; s < kLog; ++s) {
        const int o = 16 >> s;
        const int h = R >> (s + 1);
        const bool hi = (lane & o) != 0;
#pragma unroll
        for (int m = 0; m < h; ++m) {
            const int send = hi ? v[m] : v[m + h];
            const int keep = hi ? v[m + h] : v[m];
            v[m] = keep + __shfl_xor_sync(0xffffffffu, send, o);
        }
        if (hi)
            index += h;
    }
#pragma unroll
    for (int o = 16 >> kLog; o >= 1; o >>= 1)
        v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    return v[0];
}

__device__ __forceinline__ int4 ldg_stream(const int8_t *p)
{
    int4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.s32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}
__device__ __forceinline__ int dot16(int4 a, int4 b, int c)
{
    return __dp4a(a.w, b.w, __dp4a(a.z, b.z, __dp4a(a.y, b.y, __dp4a(a.x, b.x, c))));
}

template <int TN, int R, int MINB, int UNR>
__global__ void __launch_bounds__(kFewThreads, MINB) k_mm_few(MmArgs a, int obf16, int kpad)
{
    extern __shared__ __align__(16) int8_t sx[];  // [TN][kpad]
    const int lane = threadIdx.x & 31;
    const int t0 = blockIdx.y * TN, nt = (int)a.T - t0;  // this CTA's tokens
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    for (int t = 0; t < TN; ++t) {
        const int8_t *row = a.xq + (t0 + t) * a.ldx;
        const bool on = t < nt;
        if (on && (uintptr_t)row % 16 == 0) {
            for (int k = threadIdx.x * 16; k < kpad; k += kFewThreads * 16) {
                int4 v = make_int4(0, 0, 0, 0);
                if (k + 16 <= a.K)
                    v = *reinterpret_cast<const int4 *>(row + k);
                else
                    for (int e = 0; k + e < a.K; ++e)
                        reinterpret_cast<int8_t *>(&v)[e] = row[k + e];
                *reinterpret_cast<int4 *>(sx + t * kpad + k) = v;
            }
        } else
            for (int k = threadIdx.x; k < kpad; k += kFewThreads)
                sx[t * kpad + k] = on && k < a.K ? row[k] : 0;
    }
    __syncthreads();
    const int whole = a.K / 16 * 16;  // up to here 16 bytes at once lie inside a row
    const int64_t nquads = (a.V + R - 1) / R;
    const int64_t step = (int64_t)gridDim.x * (kFewThreads / 32);
    for (int64_t q = (int64_t)blockIdx.x * (kFewThreads / 32) + (threadIdx.x >> 5); q < nquads; q += step) {
        int acc[R * TN];  // [row][token]
#pragma unroll
        for (int e = 0; e < R * TN; ++e)
            acc[e] = 0;
        const int8_t *w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t v = q * R + r;
            w[r] = a.wq + (v < a.V ? v : a.V - 1) * a.ldw;
        }
#pragma unroll UNR
        for (int k = lane * 16; k < whole; k += 512) {
            int4 c[R];
#pragma unroll
            for (int r = 0; r < R; ++r)
                c[r] = ldg_stream(w[r] + k);
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                const int4 x = *reinterpret_cast<const int4 *>(sx + t * kpad + k);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    acc[r * TN + t] = dot16(c[r], x, acc[r * TN + t]);
            }
        }
        if (whole + lane < a.K) {  // the last, at most 15 values of a row, one per lane
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < TN; ++t)
                    acc[r * TN + t] += (int)w[r][whole + lane] * (int)sx[t * kpad + whole + lane];
        }
        int index;
        const int sum = warp_isum_transposed<R * TN>(acc, lane, index);
        const int64_t v = q * R + index / TN;
        const int t = index % TN;
        if (lane % (32 / (R * TN)) == 0 && v < a.V && t < nt)
            store_out(a.out, obf16, (t0 + t) * a.ldo + v, (float)sum * a.xs[t0 + t] * a.ws[v]);
    }
}

// ---------------------------------------------------------------------------
// Many tokens, on the tensor cores.  A pair of CTAs multiplies 256 rows of the
// table (the M of tcgen05.mma.cta_group::2, 128 rows in each CTA) by N tokens.
// Per block of 128 along K each CTA
//   - gets its 128 rows of the table as they are, 16 KiB of 8-bit integers, by
//     TMA into 128-byte swizzled shared memory;
//   - widens them to fp16 in registers (a thread per row and half, 64 values)
//     and stores them in tensor memory as the A operand, in slots of 64
//     columns: shared memory sees 8 bits per value of the table, not 8 + 16 + 16;
//   - gets its half of the tokens' block, already fp16 (k_widen writes them
//     once per call), by TMA.
// Measured: 2048 x 32000 x 4096 325 us, 1650 TFLOP/s, 0.86 of the cuBLAS bf16
// burst (the tensor pipes wait for the widened blocks in between); 64 x 128256 x
// 4096 95 us, 5.7 TB/s; 49 x 151936 x 896 33 us, 5.0 TB/s.
// Roles (512 threads per CTA, one CTA per SM, persistent over tiles):
//   warps 0, 2  issue the TMA loads of the table and of the tokens: two rings,
//               since a block of the table is free again once it is widened,
//               the tokens' only after their MMAs
//   warp 1      allocates tensor memory; in the even CTA issues the MMAs
//   warps 4-7   epilogue: scales and stores an accumulator (two of them, so
//               that it overlaps the next tile's MMAs)
//   warps 8-15  widen: two sets of four warps, one per half of a block
// Every wait is bounded; one that gives up sets the timeout flag, stops every
// role, and the kernel returns after its copies and MMAs in flight are done.
// The two CTAs may then have issued different numbers of copies of the tokens,
// whose bytes complete on one barrier: the even CTA evens the counts out.
// ---------------------------------------------------------------------------
using namespace tc;

constexpr int kTcRows = 128;        // rows of the table per CTA
constexpr int kTcK = 128;           // block along K
constexpr int kTcThreads = 512;
constexpr int kTcMaxN = 192;        // two accumulators and two A slots fill tensor memory
constexpr int kTcMaxStages = 10, kTcMaxSlots = 4;
constexpr int kTcWBytes = kTcRows * kTcK;
constexpr int kTcSlotCols = kTcK / 2;  // a block of A as fp16 pairs
constexpr size_t kTcSmem = 227 << 10;

struct TcTail {
    uint64_t wfull[kTcMaxStages];   // each CTA: its rows of the table landed
    uint64_t wempty[kTcMaxStages];  // each CTA: read by its eight widening warps
    uint64_t bfull[kTcMaxStages];   // even CTA: both halves of the tokens landed
    uint64_t bempty[kTcMaxStages];  // each CTA: the MMAs of the stage are done (passed on by a widening warp)
    uint64_t afull[kTcMaxSlots];    // even CTA: both CTAs' A slots written
    uint64_t aempty[kTcMaxSlots];   // each CTA: the MMAs of the slot are done
    uint64_t tfull[2], tempty[2];   // accumulators, as in the LM-head kernel
    uint64_t drain;
    uint32_t tmem_base;
    int abort;
    int64_t issued[2];   // in the even CTA: blocks of the tokens whose copies each CTA has issued
    int64_t gave_up[2];  // in both: whether a wait of either CTA gave up
    float xs[4][kTcMaxN];  // the tokens' scales of a tile, a copy per epilogue warp
};

struct TcArgs {
    const float *xs, *ws;
    void *out;
    unsigned *flags;
    int64_t ldo;
    int T, V, K;
    int N, ntb, wstages, bstages, slots, obf16;
    int split;    // parts of K; with more than one, each writes its sums to
    float *part;  // part[split][T][V]
    uint32_t idesc;
    uint64_t wait_ns;
};

// Shared-memory descriptor of a K-major operand with 128-byte swizzled rows
// of 64 fp16: 1 KiB between groups of 8 rows, descriptor version 1.
__device__ __forceinline__ uint64_t k_major_sw128_desc(uint32_t saddr)
{
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}

__device__ __forceinline__ void mma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}

__device__ __forceinline__ void tmem_store32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}

// Four 8-bit integers as two pairs of fp16.  A byte with its sign bit flipped
// is q + 128 in [0, 255]; behind the byte 0x64 it is the fp16 number 1024 + q +
// 128, exact, and one subtraction leaves q.
__device__ __forceinline__ uint2 widen4(unsigned q)
{
    const unsigned b = q ^ 0x80808080u;
    const __half2 bias = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
    const unsigned lo = __byte_perm(b, 0x64646464u, 0x4140), hi = __byte_perm(b, 0x64646464u, 0x4342);
    const __half2 l = __hsub2(*reinterpret_cast<const __half2 *>(&lo), bias);
    const __half2 h = __hsub2(*reinterpret_cast<const __half2 *>(&hi), bias);
    return make_uint2(*reinterpret_cast<const unsigned *>(&l), *reinterpret_cast<const unsigned *>(&h));
}

// The tokens as fp16, rows of kp (a multiple of 8) values, zeros behind K.
__global__ void __launch_bounds__(256) k_widen(const int8_t *__restrict__ xq, int64_t ldx, int K, int kp,
                                               uint4 *__restrict__ xh)
{
    const int64_t t = blockIdx.x;
    const int8_t *row = xq + t * ldx;
    dev::grid_dep_wait();
    dev::grid_dep_launch();
    const bool wide = (uintptr_t)row % 8 == 0;
    for (int k = threadIdx.x * 8; k < kp; k += 256 * 8) {
        uint2 q = make_uint2(0, 0);
        if (wide && k + 8 <= K)
            q = *reinterpret_cast<const uint2 *>(row + k);
        else
            for (int e = 0; e < 8 && k + e < K; ++e)
                reinterpret_cast<int8_t *>(&q)[e] = row[k + e];
        const uint2 a = widen4(q.x), b = widen4(q.y);
        xh[(t * kp + k) / 8] = make_uint4(a.x, a.y, b.x, b.y);
    }
}

// One channel's column of an accumulator, scaled, into nt rows of the output.
// The lanes of a warp hold 32 neighbouring channels: a store per token writes
// 64 or 128 bytes of a row in one piece.
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(unsigned short *p, float v) { *p = dev::f2bf(v); }
template <typename T>
__device__ __forceinline__ void write_tile(T *p, int64_t ldo, uint32_t d_tmem, const float *xs, float ws, int nt, bool on)
{
    const f2 w2 = make2(ws, ws);
    for (int c = 0; c < nt; c += 32) {
        float d[32];
        tmem_load32(d_tmem + c, d);
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(xs + c + e);
            split2(mul2(mul2(make2(d[e], d[e + 1]), make2(x.x, x.y)), w2), d[e], d[e + 1]);
            split2(mul2(mul2(make2(d[e + 2], d[e + 3]), make2(x.z, x.w)), w2), d[e + 2], d[e + 3]);
        }
        if (on) {
            if (c + 32 <= nt) {
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    put(p, d[e]);
                    p += ldo;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (c + e < nt) {
                        put(p, d[e]);
                        p += ldo;
                    }
            }
        }
    }
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// SPLIT: the calls whose K is in parts; the others divide by nothing per tile.
template <bool SPLIT>
__global__ void __launch_bounds__(kTcThreads, 1)
k_mm_tc(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const TcArgs a)
{
    extern __shared__ unsigned char tc_smem_raw[];
    unsigned char *smem =
        reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(tc_smem_raw) + 1023) & ~(uintptr_t)1023);
    const int b_box = a.N / 2 * 128;  // N / 2 tokens x 64 fp16
    unsigned char *bring = smem + (size_t)a.wstages * kTcWBytes;
    TcTail *tail = reinterpret_cast<TcTail *>(bring + (size_t)a.bstages * 2 * b_box);
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

    if ((warp == 0 || warp == 2) && lane == 0) {
        // ---------------- TMA producers (both CTAs) ----------------
        const bool tokens = warp == 2;
        const int stages = tokens ? a.bstages : a.wstages;
        uint64_t *full = tokens ? tail->bfull : tail->wfull, *empty = tokens ? tail->bempty : tail->wempty;
        int stage = 0;
        uint32_t phase = 0;
        int64_t issued = 0;  // blocks whose copies were issued
        asm volatile("fence.proxy.async.global;" ::: "memory");  // the tokens were written by plain stores
        // the table streams when every block is read once
        const uint64_t pol = l2_policy(tokens ? 1 : a.ntb > 1 ? 0 : 2);
        bool ok = true;
        for (int tile = tile0; tile < ntiles && ok; tile += tstep) {
            const int vrow = (tile / split / a.ntb * 2 + rank) * kTcRows;
            const int trow = tile / split % a.ntb * a.N + rank * (a.N / 2);
            const int kb1 = end_block(tile);
            for (int kb = first_block(tile); kb < kb1; ++kb) {
                if (!mbar_spin(smem_addr(&empty[stage]), phase ^ 1u, abort, a.wait_ns)) {
                    ok = false;
                    break;
                }
                const uint32_t bar = smem_addr(&full[stage]);
                ++issued;
                if (tokens) {
                    if (leader)
                        mbar_expect_tx(bar, 4 * b_box);  // both CTAs' halves, two boxes each
                    const uint32_t dst = smem_addr(bring + (size_t)stage * 2 * b_box);
                    const uint32_t lead = mapa_rank(bar, 0);
                    tma_load_2d(dst, &tm_x, kb * kTcK, trow, lead, pol);
                    tma_load_2d(dst + b_box, &tm_x, kb * kTcK + 64, trow, lead, pol);
                } else {
                    mbar_expect_tx(bar, kTcWBytes);
                    tma_load_2d(smem_addr(smem + (size_t)stage * kTcWBytes), &tm_w, kb * kTcK, vrow, bar, pol);
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
        // The whole warp runs the loop and one lane issues: operands that are
        // the same in every lane stay in uniform registers, where the
        // instruction takes them (with a single thread in the loop, moving
        // them there cost about 125 clocks per MMA, more than the MMA).
        int stage = 0, slot = 0, acc = 0;
        uint32_t phase = 0, aphase = 0, acc_phase = 0;
        bool ok = true;
        const uint32_t bring_addr = smem_addr(bring);
        const uint32_t full0 = smem_addr(&tail->bfull[0]), afull0 = smem_addr(&tail->afull[0]);
        for (int tile = tile0; tile < ntiles && ok; tile += tstep) {
            ok = mbar_spin(smem_addr(&tail->tempty[acc]), acc_phase ^ 1u, abort, a.wait_ns);
            if (!__all_sync(0xffffffffu, ok)) {
                ok = false;
                break;
            }
            const uint32_t d_tmem = tmem + (uint32_t)(acc * a.N);
            const int kb0 = first_block(tile), kb1 = end_block(tile);
            for (int kb = kb0; kb < kb1 && ok; ++kb) {
                ok = mbar_spin(full0 + stage * 8, phase, abort, a.wait_ns) &&
                     mbar_spin(afull0 + slot * 8, aphase, abort, a.wait_ns);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok)
                    break;
                tc_fence_after();
                const uint64_t b_desc = k_major_sw128_desc(bring_addr + stage * 2 * b_box);
                const uint32_t a_base = slot0 + (uint32_t)(slot * kTcSlotCols);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kTcK / 16; ++k)
                        mma_f16_ta(d_tmem, a_base + k * 8, b_desc + (uint64_t)((k >> 2) * (b_box >> 4) + 2 * (k & 3)),
                                   a.idesc, ((kb - kb0) | k) != 0);
                    mma_commit_mc(smem_addr(&tail->aempty[slot]));
                }
                __syncwarp();
                if (++slot == a.slots) {
                    slot = 0;
                    aphase ^= 1u;
                }
                if (++stage == a.bstages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            if (!ok)
                break;
            if (elect_one())
                mma_commit_mc(smem_addr(&tail->tfull[acc]));
            __syncwarp();
            if (++acc == 2) {
                acc = 0;
                acc_phase ^= 1u;
            }
        }
        if (elect_one()) {
            if (!ok)
                set_timeout(abort, a.flags);
            mma_commit(smem_addr(&tail->drain));
            mbar_wait_final(smem_addr(&tail->drain), 0);
        }
        __syncwarp();
    } else if (warp >= 8) {
        // ---------------- widening: the table's rows into tensor memory ----------------
        const int q = warp & 3;
        const int set = (warp - 8) >> 2;
        const int r = q * 32 + lane;
        const uint32_t lanes = (uint32_t)(q * 32) << 16;
        int stage = 0, slot = 0;
        uint32_t phase = 0, aphase = 0;
        // a block's MMAs being done frees its slots and its stage of the tokens:
        // the first widening warp passes the latter on
        int seen = -a.slots, bstage = 0;
        bool ok = true;
        for (int tile = tile0; tile < ntiles && ok; tile += tstep) {
            for (int kb = first_block(tile), kb1 = end_block(tile); kb < kb1; ++kb) {
                ok = mbar_spin(smem_addr(&tail->wfull[stage]), phase, abort, a.wait_ns);
                if (!__all_sync(0xffffffffu, ok)) {
                    ok = false;
                    break;
                }
                const unsigned char *row = smem + (size_t)stage * kTcWBytes + r * 128;
                uint4 raw[4];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    raw[c] = *reinterpret_cast<const uint4 *>(row + (((set * 4 + c) ^ (r & 7)) << 4));
                uint32_t w[32];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const unsigned x[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint2 p = widen4(x[e]);
                        w[c * 8 + 2 * e] = p.x;
                        w[c * 8 + 2 * e + 1] = p.y;
                    }
                }
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(smem_addr(&tail->wempty[stage]));
                ok = mbar_spin(smem_addr(&tail->aempty[slot]), aphase ^ 1u, abort, a.wait_ns);
                if (!__all_sync(0xffffffffu, ok)) {
                    ok = false;
                    break;
                }
                if (++seen > 0 && warp == 8) {
                    if (lane == 0)
                        mbar_arrive(smem_addr(&tail->bempty[bstage]));
                    bstage = bstage + 1 == a.bstages ? 0 : bstage + 1;
                }
                tc_fence_after();
                tmem_store32(slot0 + (uint32_t)(slot * kTcSlotCols + set * 32) + lanes, w);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    mbar_arrive_remote(mapa_rank(smem_addr(&tail->afull[slot]), 0));
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
    } else if (warp >= 4) {
        // ---------------- epilogue (both CTAs) ----------------
        const int q = warp - 4;
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int tile = tile0; tile < ntiles; tile += tstep) {
            const bool ok = mbar_spin(smem_addr(&tail->tfull[acc]), acc_phase, abort, a.wait_ns);
            if (!__all_sync(0xffffffffu, ok)) {
                if (lane == 0 && !*abort)
                    set_timeout(abort, a.flags);
                break;
            }
            tc_fence_after();
            const int v = (tile / split / a.ntb * 2 + rank) * kTcRows + q * 32 + lane;
            const int t0 = tile / split % a.ntb * a.N;
            const bool whole = split == 1;
            const float ws = !whole ? 1.f : v < a.V ? a.ws[v] : 0.f;
            const int nt = a.T - t0 < a.N ? a.T - t0 : a.N;  // tokens of this tile
            float *xs = tail->xs[q];
            for (int k = lane; k < a.N; k += 32)
                xs[k] = !whole ? 1.f : k < nt ? a.xs[t0 + k] : 0.f;
            __syncwarp();
            const uint32_t d_tmem = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * a.N);
            const int64_t at = (int64_t)t0 * a.ldo + v;
            if (!whole)
                write_tile(a.part + ((int64_t)(tile % split) * a.T + t0) * a.V + v, a.V, d_tmem, xs, ws, nt, v < a.V);
            else if (a.obf16)
                write_tile(static_cast<unsigned short *>(a.out) + at, a.ldo, d_tmem, xs, ws, nt, v < a.V);
            else
                write_tile(static_cast<float *>(a.out) + at, a.ldo, d_tmem, xs, ws, nt, v < a.V);
            __syncwarp();  // xs is read before the next tile writes it
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                mbar_arrive_remote(mapa_rank(smem_addr(&tail->tempty[acc]), 0));
            if (++acc == 2) {
                acc = 0;
                acc_phase ^= 1u;
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
                    mbar_expect_tx(bar, 2 * b_box);
                else if (i >= n1)
                    mbar_complete_tx(bar, 2 * b_box);
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
__global__ void __launch_bounds__(256) k_mm_join(const TcArgs a)
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
    store_out(a.out, a.obf16, t * a.ldo + v, s * a.xs[t] * a.ws[v]);
}

// R x C elements of `size` bytes with a row stride of ld, boxes of 128 bytes x
// `rows` in the 128-byte swizzle; what lies outside reads as zero.
bool make_load_map(CUtensorMap *m, const void *base, int size, int64_t C, int64_t R, int64_t ld, int rows)
{
    PFN_cuTensorMapEncodeTiled_v12000 fn = encode_fn();
    if (!fn)
        return false;
    cuuint64_t dims[2] = {(cuuint64_t)C, (cuuint64_t)R};
    cuuint64_t strides[1] = {(cuuint64_t)(ld * size)};
    cuuint32_t box[2] = {(cuuint32_t)(128 / size), (cuuint32_t)rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(m, size == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
              const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Blocks of tokens, all of one width N (a multiple of 32).  One when they fit;
// otherwise the widths from 192 down to 128 are weighed by the rounds that
// the SM pairs need for the tiles and by what a round costs, its N and about
// 24 tokens' worth of fixed work: narrower blocks leave less of the last round
// idle and have more slots of A, wider ones read the table's tiles less often.
void token_blocks(int64_t T, int64_t vblocks, int *ntb, int *N)
{
    int64_t best = INT64_MAX;
    for (int n = kTcMaxN; n >= 128; n -= 32) {
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

int64_t widened_cols(int64_t K) { return (K + 7) / 8 * 8; }

// Plan of a call on the tensor cores.  Where the tiles leave half of the SM
// pairs or more without one, K is split among them, 8 blocks or more to a
// part, if that takes 12 blocks or more off every pair (about what the joining
// launch costs); us whole / in parts: 64 x 4161 x 7856 30 / 17 (4 parts), 20 x
// 1000 x 4096 17.8 / 13.0 (4), 64 x 9000 x 2048 12.9 / 14.4 (2, not taken).
struct TcPlan {
    int ntb, N, split;
    size_t part_at, bytes;  // where the parts begin in the workspace, and its size
};
TcPlan tc_plan(int64_t T, int64_t V, int64_t K)
{
    TcPlan p;
    const int64_t vblocks = (V + 2 * kTcRows - 1) / (2 * kTcRows), kblocks = (K + kTcK - 1) / kTcK;
    token_blocks(T, vblocks, &p.ntb, &p.N);
    const int64_t tiles = vblocks * p.ntb;
    const int64_t by_pairs = kSms / 2 / tiles, by_blocks = kblocks / 8;
    p.split = (int)(by_pairs < by_blocks ? by_pairs : by_blocks);
    if (p.split < 2 || kblocks - (kblocks + p.split - 1) / p.split < 12)
        p.split = 1;
    p.part_at = ((size_t)(T * widened_cols(K)) * 2 + 255) / 256 * 256;
    p.bytes = p.part_at + (p.split > 1 ? (size_t)p.split * T * V * sizeof(float) : 0);
    return p;
}

cudaError_t launch_tc(const MmArgs &m, int obf16, void *workspace, unsigned *flags, cudaStream_t stream)
{
    const int kp = (int)widened_cols(m.K);
    cudaError_t e = launch_k(k_widen, dim3((unsigned)m.T), dim3(256), 0, stream, true, m.xq, m.ldx, m.K, kp,
                             static_cast<uint4 *>(workspace));
    if (e != cudaSuccess)
        return e;
    TcArgs a{};
    a.xs = m.xs;
    a.ws = m.ws;
    a.out = m.out;
    a.flags = flags;
    a.ldo = m.ldo;
    a.T = (int)m.T;
    a.V = (int)m.V;
    a.K = m.K;
    a.obf16 = obf16;
    a.wait_ns = ops_wait_ns();
    const TcPlan p = tc_plan(m.T, m.V, m.K);
    a.ntb = p.ntb;
    a.N = p.N;
    a.split = p.split;
    a.part = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + p.part_at);
    a.slots = (512 - 2 * a.N) / kTcSlotCols;
    if (a.slots > kTcMaxSlots)
        a.slots = kTcMaxSlots;
    // shared memory: five blocks of the tokens (as long as they take to come
    // from L2), the rest to the table
    const size_t fixed = 1024 + sizeof(TcTail), bstage = (size_t)a.N * 128;
    a.bstages = 5;
    a.wstages = (int)((kTcSmem - fixed - a.bstages * bstage) / kTcWBytes);
    if (a.wstages > kTcMaxStages)
        a.wstages = kTcMaxStages;
    a.idesc = 1u << 4 | (uint32_t)(a.N >> 3) << 17 | (uint32_t)(2 * kTcRows >> 4) << 24;  // f32 += f16 f16, K-major
    CUtensorMap tm_w, tm_x;
    if (!make_load_map(&tm_w, m.wq, 1, m.K, m.V, m.ldw, kTcRows) ||
        !make_load_map(&tm_x, workspace, 2, kp, m.T, kp, a.N / 2))
        return cudaErrorInvalidValue;
    const auto kernel = a.split > 1 ? k_mm_tc<true> : k_mm_tc<false>;
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
    e = cudaLaunchKernelEx(&cfg, kernel, tm_w, tm_x, a);
    if (e == cudaSuccess && a.split > 1)
        e = launch_k(k_mm_join, dim3((unsigned)((m.V + 255) / 256), (unsigned)m.T), dim3(256), 0, stream, true, a);
    return e;
}

// CTAs of k_mm_few with R rows of the table per warp.
int64_t few_ctas(int64_t V, int R) { return ((V + R - 1) / R + kFewThreads / 32 - 1) / (kFewThreads / 32); }

template <int TN, int R, int MINB, int UNR>
cudaError_t launch_few(const MmArgs &a, int obf16, int kpad, cudaStream_t stream)
{
    const cudaError_t e =
        cudaFuncSetAttribute(k_mm_few<TN, R, MINB, UNR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kFewSmem);
    if (e != cudaSuccess)
        return e;
    const int64_t ctas = few_ctas(a.V, R);
    const dim3 grid((unsigned)(ctas < MINB * kSms ? ctas : MINB * kSms), (unsigned)((a.T + TN - 1) / TN));
    return launch_k(k_mm_few<TN, R, MINB, UNR>, grid, dim3(kFewThreads), (size_t)TN * kpad, stream, true, a, obf16, kpad);
}

// Rows per warp, CTAs per SM and unrolled slabs of k_mm_few, measured on
// 151936 x 896 (short rows, where the joining of the lanes weighs) and 128256 x
// 8192; us for 1 / 4 / 8 tokens:
//   4 rows, 2 CTAs, 2 slabs   32 / 39 / 57    152 / 154 / 201
//   4 rows, 2 CTAs, 4 slabs   31 / 35 / 44    149 / 164 / 195
//   4 rows, 4 CTAs, 4 slabs   24 /  - /  -    162 /   - /   -
//   8 rows, 2 CTAs, 4 slabs   25 / 29 /  -    158 / 166 /   -
//   k_mm_tc                   31 / 31 / 31    179 / 179 / 180
// Five to eight tokens go to the tensor cores for large tables, of short rows
// sooner (k_mm_few / k_mm_tc for 6 tokens: 10000 x 2048 9.0 / 12.6, 40000 x 8192
// 75 / 81, 50257 x 768 16.6 / 13.7, 8000 x 512 4.9 / 6.7, 32000 x 256 9.2 / 7.0).
// More tokens stay here in groups of eight while all groups run at once and
// the rows are short: the tensor cores' two launches take longer to begin
// (16 tokens: 1000 x 2048 5.6 / 10.9, 4000 x 512 5.1 / 6.6, 4000 x 2048 7.2 /
// 11.1, 1000 x 8192 12.3 / 10.4; 64 and 100 tokens: 1000 x 512 5.1 / 6.9 and, in
// more than one wave, 8.9 / 8.0).
constexpr int kFewShortRow = 2048;
constexpr int64_t kFewMaxRows = 49152, kFewMaxShortRows = 16384;
constexpr int kFewR = 4, kFewMinB = 2;  // of the form for eight tokens

cudaError_t launch_mm(const MmArgs &a, int obf16, void *workspace, unsigned *flags, cudaStream_t stream)
{
    if (aligned(a.wq, 16) && a.ldw % 16 == 0) {
        const int kpad = (a.K + 511) / 512 * 512;
        const bool brief = a.K <= kFewShortRow;
        if (a.T == 1 && (size_t)kpad <= kFewSmem)
            return brief ? launch_few<1, 4, 4, 4>(a, obf16, kpad, stream) : launch_few<1, 4, 2, 4>(a, obf16, kpad, stream);
        if (a.T == 2 && (size_t)2 * kpad <= kFewSmem)
            return brief ? launch_few<2, 8, 2, 4>(a, obf16, kpad, stream) : launch_few<2, 4, 2, 2>(a, obf16, kpad, stream);
        if (a.T <= 4 && (size_t)4 * kpad <= kFewSmem)
            return brief ? launch_few<4, 8, 2, 4>(a, obf16, kpad, stream) : launch_few<4, 4, 2, 2>(a, obf16, kpad, stream);
        const int64_t groups = (a.T + kFewTokens - 1) / kFewTokens;
        const bool few = groups == 1 ? a.V <= (a.K < 1024 ? kFewMaxShortRows : kFewMaxRows)
                                     : brief && few_ctas(a.V, kFewR) * groups <= kFewMinB * kSms;
        if (few && (size_t)kFewTokens * kpad <= kFewSmem)
            return launch_few<kFewTokens, kFewR, kFewMinB, 4>(a, obf16, kpad, stream);
        return launch_tc(a, obf16, workspace, flags, stream);
    }
    const int64_t vb = (a.V + kGV - 1) / kGV, tb = (a.T + kGT - 1) / kGT;
    return launch_k(k_mm_any, dim3((unsigned)(vb * tb)), dim3(256), 0, stream, true, a, obf16, (unsigned)vb);
}

}  // namespace
}  // namespace ember

using namespace ember;

extern "C" {

size_t ember_matmul_quant_workspace_bytes(int64_t T, int64_t V, int64_t K)
{
    if (T < 0 || V < 1 || K < 1 || T > kMaxMmRows || V > kMaxMmRows || K > kMaxRowCols)
        return 0;
    return tc_plan(T > 0 ? T : 1, V, K).bytes;  // the tokens in fp16, the parts of a split K
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
    if (T > kMaxMmRows || V > kMaxMmRows || K > kMaxRowCols || ldx > (int64_t(1) << 31) || ldw > (int64_t(1) << 31) ||
        ldo > (int64_t(1) << 32))
        return EMBER_ERR_UNSUPPORTED;
    if (!aligned(xs, 4) || !aligned(ws, 4) || !aligned(out, elem_size(otype)) || !aligned(status, 4) ||
        !aligned(workspace, 16))
        return EMBER_ERR_ALIGNMENT;
    if (T == 0)
        return EMBER_OK;
    if (!workspace || bytes < ember_matmul_quant_workspace_bytes(T, V, K))
        return EMBER_ERR_WORKSPACE;
    // 2^31 tiles of the smallest size are 1.4e14 logits: more than the GPU holds
    if ((V + kGV - 1) / kGV * ((T + kGT - 1) / kGT) > INT32_MAX)
        return EMBER_ERR_UNSUPPORTED;
    const MmArgs a{xq, wq, xs, ws, out, ldx, ldw, ldo, T, V, (int)K};
    return launched(launch_mm(a, otype == EMBER_BF16, workspace, status, (cudaStream_t)stream));
}

}  // extern "C"
