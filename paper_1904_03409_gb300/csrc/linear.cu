// linear.cu -- a linear layer with its epilogue, y = act(x W^T + bias) + residual, its backward,
// and their C ABI (include/stacklstm.h, stacklstm_linear_*).
//
// x [R][K], W [N][K]. With pre = x W^T + bias and dz = dy act'(pre) the backward is
//   dx = dz W (+ add),  dW = dz^T x,  dbias = the column sums of dz.
// All three contractions run on the tensor cores (tcgen05, bf16 operands, fp32 accumulators in
// tensor memory) in one kernel, gemm_parts: D [M][N] = sum over pairs (i, j) of A_i B_j^T, where
// an operand is one bf16 tensor or several parts of an fp32 one. An fp32 number is the sum of
// three bf16 numbers (8 + 8 + 8 significant bits), so the product of two has the six partial
// products of order <= 2 (what is left out is below 2^-23 of it), and of one with a bf16 number
// three: fp32 results at a sixth or a third of the bf16 tensor rate, where the CUDA cores have
// about a thirtieth of it. Operands are read by TMA as they lie, the contraction along their
// rows (K-major) or across them (MN-major), so nothing is transposed:
//   forward  A = x   [R][K] K-major    B = W  [N][K] K-major     (few rows: A = W, B = x)
//   dx       A = dz  [R][N] K-major    B = W  [N][K] MN-major
//   dW       A = dz  [R][N] MN-major   B = x  [R][K] MN-major
// dz is written once, as three bf16 parts, with the column sums of dbias.
#include <cuda.h>
#include <cudaTypedefs.h>

#include "op.cuh"
#include "tc.cuh"

namespace sl {
namespace {

using tc::smem_u32;

enum { kActNone = 0, kActRelu, kActTanh, kActGelu, kActSilu, kActs };

__device__ __forceinline__ float act_f(float z, int act)
{
    switch (act) {
    case kActRelu: return z > 0.0f || isnan(z) ? z : 0.0f;
    case kActTanh: return tanhf(z);
    case kActGelu: return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    case kActSilu: return z / (1.0f + expf(-z));
    default: return z;
    }
}
__device__ __forceinline__ float act_grad(float z, int act)
{
    switch (act) {
    case kActRelu: return z > 0.0f ? 1.0f : 0.0f;
    case kActTanh: {
        const float t = tanhf(z);
        return 1.0f - t * t;
    }
    case kActGelu: return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * expf(-0.5f * z * z) * 0.39894228f;
    case kActSilu: {
        const float s = 1.0f / (1.0f + expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    default: return 1.0f;
    }
}

// ------------------------------------------------------------------ operands
// fp32 v as the sum of three bf16 numbers, each what is left rounded to nearest, so that the parts
// are at most 1, 2^-8 and 2^-16 of v; a value that is not finite is in the first alone, and one
// that rounding would make infinite (as would its first two parts' sum) is cut towards zero.
__device__ __forceinline__ void split3(float v, __nv_bfloat16 (&p)[3])
{
    const bool finite = fabsf(v) <= 3.402823466e38f;
    p[0] = __float2bfloat16(v);
    const bool over = finite && __hisinf(p[0]);
    if (over) p[0] = __float2bfloat16_rz(v);
    const float r1 = v - __bfloat162float(p[0]);
    p[1] = !finite ? __float2bfloat16(0.0f) : over ? __float2bfloat16_rz(r1) : __float2bfloat16(r1);
    p[2] = finite ? __float2bfloat16(r1 - __bfloat162float(p[1])) : __float2bfloat16(0.0f);
}

// out [parts][rows][ld] from src [rows][cols]: the parts of fp32 numbers, or (bf16) a copy whose
// rows start on 16 bytes.
template <typename T>
__global__ void __launch_bounds__(256)
pack_parts(size_t rows, int cols, int ld, const T *__restrict__ src, __nv_bfloat16 *__restrict__ out)
{
    const size_t n = rows * cols, plane = rows * ld;
    for (size_t e = blockIdx.x * (size_t)256 + threadIdx.x; e < n; e += (size_t)gridDim.x * 256) {
        const size_t r = e / cols, c = e - r * cols, o = r * ld + c;
        if constexpr (sizeof(T) == 4) {
            __nv_bfloat16 p[3];
            split3(src[e], p);
#pragma unroll
            for (int i = 0; i < 3; ++i) out[i * plane + o] = p[i];
        } else {
            out[o] = src[e];
        }
    }
}

constexpr int kDzCols = 256, kDzRows = 64;

// dz = dy act'(pre) as three parts [3][rows][ld], and this CTA's column sums of it over its rows,
// part [row blocks][N]. A thread takes one column.
template <typename T>
__global__ void __launch_bounds__(kDzCols)
dz_parts(int rows, int N, int ld, int act, const float *__restrict__ dy, const T *__restrict__ pre,
         __nv_bfloat16 *__restrict__ out, float *__restrict__ part)
{
    const int c = blockIdx.y * kDzCols + threadIdx.x;
    if (c >= N) return;
    const int r0 = blockIdx.x * kDzRows, r1 = min(rows, r0 + kDzRows);
    const size_t plane = (size_t)rows * ld;
    float sum = 0.0f;
    for (int r = r0; r < r1; ++r) {
        float v = dy[(size_t)r * N + c];
        if (act != kActNone) v = __fmul_rn(v, act_grad(to_f32(pre[(size_t)r * N + c]), act));  // (not fused with the sum)
        sum += v;
        if (out) {
            __nv_bfloat16 p[3];
            split3(v, p);
#pragma unroll
            for (int i = 0; i < 3; ++i) out[i * plane + (size_t)r * ld + c] = p[i];
        }
    }
    if (part) part[(size_t)blockIdx.x * N + c] = sum;
}

// out[c] = the sum over s of part[s][c]: warp w adds parts w, w + 8, ..., then the eight in order.
__global__ void __launch_bounds__(256)
sum_parts(const float *__restrict__ part, int n, int N, float *__restrict__ out)
{
    __shared__ float sm[8][32];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const size_t c = blockIdx.x * (size_t)32 + lane;
    float acc = 0.0f;
    if (c < (size_t)N) {
#pragma unroll 8
        for (int s = w; s < n; s += 8) acc += part[(size_t)s * N + c];
    }
    sm[w][lane] = acc;
    __syncthreads();
    if (w == 0 && c < (size_t)N) {
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += sm[i][lane];
        out[c] = v;
    }
}

// ------------------------------------------------------------------ the contraction
// What happens to the sums of output (r, n), r a row of y / dx / dW and n a column.
struct Epilogue {
    int rows, cols;         // extents of the output
    int act;                // forward: the activation
    int bf16_out;           // forward: type of y, pre, residual
    const float *bias;      // forward [cols] or null
    const void *residual;   // forward [rows][cols] or null
    void *y, *pre;          // forward
    const float *add;       // gradients: [rows][cols] or null
    float *out;             // gradients (null: forward)
    float *part;            // split contraction: [split][rows][cols] sums, or null
};

struct GemmArgs {
    int chunks;             // 64-wide chunks of the contraction
    int npair;
    uint8_t pa[6], pb[6];   // parts of each partial product
    int split, S;           // splits of the chunks; ring stages
    int swapped;            // the output's rows are B's rows (few rows: A = W)
    Epilogue ep;
    long long limit;
    int32_t *err;
};

__device__ __forceinline__ void finish(const Epilogue &ep, int r, int n, float v)
{
    const size_t at = (size_t)r * ep.cols + n;
    if (ep.out) {
        ep.out[at] = ep.add ? v + ep.add[at] : v;
        return;
    }
    if (ep.bias) v += ep.bias[n];
    float o = act_f(v, ep.act);
    if (ep.bf16_out) {
        if (ep.pre) ((__nv_bfloat16 *)ep.pre)[at] = __float2bfloat16(v);
        if (ep.residual) o += __bfloat162float(((const __nv_bfloat16 *)ep.residual)[at]);
        ((__nv_bfloat16 *)ep.y)[at] = __float2bfloat16(o);
    } else {
        if (ep.pre) ((float *)ep.pre)[at] = v;
        if (ep.residual) o += ((const float *)ep.residual)[at];
        ((float *)ep.y)[at] = o;
    }
}

constexpr int kGemmThreads = 192;  // warps 0-3: epilogue; 4: TMA; 5: MMA
constexpr int kMaxRing = 12;
constexpr uint32_t kTileA = 128 * 128;  // 128 rows (or 2 x 64 columns) x 64 of the contraction
constexpr long long kWaitLimit = 4000000000LL, kDrain = 4000000000LL;  // clock cycles of a bounded wait

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void *tmap, int c0, int c1, int c2, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"((uint64_t)tmap), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
        : "memory");
}

__host__ __device__ constexpr uint32_t gemm_stage(int BN) { return kTileA + (uint32_t)BN * 128u; }
__host__ __device__ constexpr uint32_t gemm_smem(int S, int BN) { return 1024 + S * gemm_stage(BN) + (2 * kMaxRing + 1) * 8 + 32; }

// One 128 x BN tile (blockIdx.x: m tile fastest within a column of tiles) over the chunks of
// split blockIdx.y. MN-major operands: blocks of 64 columns, each 64 rows of 128 bytes.
template <int BN, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_parts(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const GemmArgs g)
{
    constexpr uint32_t kStage = gemm_stage(BN);
    constexpr uint32_t kCols = BN < 32 ? 32 : BN;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int S = g.S;
    const uint32_t ring0 = smem_u32(base);
    uint64_t *full = (uint64_t *)(base + (size_t)S * kStage);
    uint64_t *empty = full + kMaxRing;
    uint64_t *done = empty + kMaxRing;
    uint32_t *tmem_slot = (uint32_t *)(done + 1);
    int *n_issued = (int *)(tmem_slot + 1);
    int *n_consumed = n_issued + 1;
    volatile int *abort = (volatile int *)(n_consumed + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int mrows = g.swapped ? g.ep.cols : g.ep.rows, mt_n = (mrows + 127) / 128;
    const int m0 = (int)(blockIdx.x % mt_n) * 128, n0 = (int)(blockIdx.x / mt_n) * BN, sp = blockIdx.y;
    const int c_lo = (int)((long long)g.chunks * sp / g.split), c_hi = (int)((long long)g.chunks * (sp + 1) / g.split);
    const int its = (c_hi - c_lo) * g.npair;
    if (tid == 0) {
        for (int s = 0; s < S; ++s) {
            tc::mbar_init(&full[s], 1);
            tc::mbar_init(&empty[s], 1);
        }
        tc::mbar_init(done, 1);
        *n_issued = 0;
        *n_consumed = 0;
        *abort = 0;
        tc::fence_mbar_init();
    }
    if (warp == 4) tc::tmem_alloc(tmem_slot, kCols);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto fail = [&]() {
        *abort = 1;
        atomicCAS(g.err, 0, (int)SL_ERR_TIMEOUT);
    };

    if (warp == 4) {
        if (lane == 0) {
            int it = 0;
            for (; it < its; ++it) {
                const int s = it % S;
                if (it >= S && !tc::mbar_wait(&empty[s], (uint32_t)(it / S - 1) & 1, g.limit, abort)) {
                    fail();
                    break;
                }
                const uint32_t st = ring0 + s * kStage;
                const int k0 = (c_lo + it / g.npair) * 64, pair = it % g.npair;
                tc::mbar_arrive_expect_tx(&full[s], kStage);
                if constexpr (A_MN) {
                    tma_load_3d(st, &tm_a, m0, k0, g.pa[pair], &full[s]);
                    tma_load_3d(st + 8192, &tm_a, m0 + 64, k0, g.pa[pair], &full[s]);
                } else {
                    tma_load_3d(st, &tm_a, k0, m0, g.pa[pair], &full[s]);
                }
                if constexpr (B_MN) {
#pragma unroll
                    for (int nb = 0; nb < BN / 64; ++nb)
                        tma_load_3d(st + kTileA + nb * 8192, &tm_b, n0 + nb * 64, k0, g.pb[pair], &full[s]);
                } else {
                    tma_load_3d(st + kTileA, &tm_b, k0, n0, g.pb[pair], &full[s]);
                }
            }
            *n_issued = it;
        }
        __syncwarp();
    } else if (warp == 5) {
        if (lane == 0) {
            constexpr uint32_t idesc = tc::idesc_bf16(BN, A_MN, B_MN);
            int it = 0;
            for (; it < its && !*abort; ++it) {
                const int s = it % S;
                if (!tc::mbar_wait(&full[s], (uint32_t)(it / S) & 1, g.limit, abort)) {
                    fail();
                    break;
                }
                tc::tc_fence_after();
                const uint32_t as = ring0 + s * kStage, bs = as + kTileA;
#pragma unroll
                for (int k = 0; k < 4; ++k)  // 16 of the contraction: 32 bytes of a row, or 16 rows
                    tc::mma_bf16(tmem, A_MN ? tc::smem_desc(as + k * 2048, 8192, 1024) : tc::smem_desc(as + k * 32, 16, 1024),
                                 B_MN ? tc::smem_desc(bs + k * 2048, 8192, 1024) : tc::smem_desc(bs + k * 32, 16, 1024),
                                 idesc, (it | k) != 0);
                tc::mma_commit(&empty[s]);
            }
            *n_consumed = it;
            tc::mma_commit(done);
        }
        __syncwarp();
    } else {
        const bool ok = tc::mbar_wait(done, 0, g.limit, nullptr);
        if (!ok) fail();
        tc::tc_fence_after();
        if (ok && !*abort) {
            const int m = m0 + warp * 32 + lane;
            const uint32_t trow = tmem + ((uint32_t)(warp * 32) << 16);
            const Epilogue &ep = g.ep;
            float *part = ep.part ? ep.part + (size_t)sp * ep.rows * ep.cols : nullptr;
#pragma unroll 1
            for (int c = 0; c < BN; c += 16) {
                float v[16];
                tc::tmem_ld16(trow + c, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int n = n0 + c + i;
                    const int r = g.swapped ? n : m, col = g.swapped ? m : n;
                    if (r < ep.rows && col < ep.cols) {
                        const float w = its ? v[i] : 0.0f;
                        if (part)
                            part[(size_t)r * ep.cols + col] = w;
                        else
                            finish(ep, r, col, w);
                    }
                }
            }
        }
    }
    __syncthreads();
    if (warp == 4 && lane == 0) {
        // copies still in flight after an abort: issued, never seen landed
        for (int it = *n_consumed; it < *n_issued; ++it)
            tc::mbar_wait(&full[it % S], (uint32_t)(it / S) & 1, kDrain, nullptr);
    }
    if (warp == 5 && lane == 0) tc::mbar_wait(done, 0, kDrain, nullptr);
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 4) tc::tmem_dealloc(tmem, kCols);
}

// The splits' sums of each output added in split order, then its epilogue.
__global__ void __launch_bounds__(256)
join_splits(const Epilogue ep, int split)
{
    const size_t n = (size_t)ep.rows * ep.cols;
    for (size_t e = blockIdx.x * (size_t)256 + threadIdx.x; e < n; e += (size_t)gridDim.x * 256) {
        float v = 0.0f;
        for (int s = 0; s < split; ++s) v += ep.part[(size_t)s * n + e];
        finish(ep, (int)(e / ep.cols), (int)(e % ep.cols), v);
    }
}

// ------------------------------------------------------------------ host side
PFN_cuTensorMapEncodeTiled_v12000 encoder(cudaError_t *e)
{
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;  // the same address for every thread that looks it up
    *e = cudaSuccess;
    if (fn) return fn;
    cudaDriverEntryPointQueryResult q;
    void *p = nullptr;
    *e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q);
    if (!*e && (q != cudaDriverEntryPointSuccess || !p)) *e = cudaErrorNotSupported;
    if (!*e) fn = (PFN_cuTensorMapEncodeTiled_v12000)p;
    return fn;
}

// An operand: parts x rows x cols bf16, rows ld apart.
struct Operand {
    const void *p;
    size_t rows;
    int cols, ld, parts;
};

// The map of an operand read in boxes of 64 columns x box_rows rows of one part, 128-byte
// swizzled; what is outside reads as zero.
cudaError_t operand_map(CUtensorMap *tm, const Operand &o, int box_rows)
{
    cudaError_t e;
    auto encode = encoder(&e);
    if (e) return e;
    const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.parts};
    const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)o.ld * 2 * o.rows};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, es[3] = {1, 1, 1};
    const CUresult r = encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(o.p), dims, strides, box, es,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int BN, bool A_MN, bool B_MN>
cudaError_t launch_gemm(const stacklstm_op *op, const Operand &a, const Operand &b, GemmArgs g, unsigned tiles)
{
    CUtensorMap ta, tb;
    cudaError_t e = operand_map(&ta, a, A_MN ? 64 : 128);
    if (!e) e = operand_map(&tb, b, B_MN ? 64 : BN);
    if (e) return e;
    g.S = std::min(kMaxRing, (int)((227 * 1024 - gemm_smem(0, BN)) / gemm_stage(BN)));
    const size_t smem = gemm_smem(g.S, BN);
    if ((e = smem_at_least((const void *)gemm_parts<BN, A_MN, B_MN>, smem))) return e;
    gemm_parts<BN, A_MN, B_MN><<<dim3(tiles, g.split), kGemmThreads, smem, op->stream>>>(ta, tb, g);
    return cudaGetLastError();
}

enum { kWsX = 0, kWsW, kWsDz, kWsSum, kWsPart };  // workspace buffers

// D = sum over the parts' products of A B^T, kcols long, and its epilogue; the contraction is
// split over more CTAs where its tiles leave SMs idle.
template <bool A_MN, bool B_MN>
cudaError_t contract(stacklstm_op *op, const Operand &a, const Operand &b, int kcols, bool swapped, Epilogue ep)
{
    GemmArgs g = {};
    g.chunks = (int)ceil_div(kcols, 64);
    for (int i = 0; i < a.parts; ++i)
        for (int j = 0; j < b.parts; ++j)
            if (i + j <= 2) {
                g.pa[g.npair] = (uint8_t)i;
                g.pb[g.npair++] = (uint8_t)j;
            }
    g.swapped = swapped;
    g.limit = kWaitLimit;
    g.err = op->err;
    const int M = swapped ? ep.cols : ep.rows, N = swapped ? ep.rows : ep.cols;
    const int bn = N <= 64 ? 64 : N <= 128 ? 128 : 256;
    const size_t tiles = (size_t)ceil_div(M, 128) * ceil_div(N, bn);
    g.split = (int)std::max<size_t>(1, std::min<size_t>(g.chunks / 4, (size_t)op->num_sms / tiles));
    // fp32 results: the tensor cores' fp32 additions cut instead of rounding, which costs about
    // 1.7e-8 of the result an addition (measured: 1e-4 after 6012 of them); no accumulator takes
    // more than 15 chunks' parts, the sums of which are added in fp32
    if (ep.out || !ep.bf16_out) g.split = std::max(g.split, std::min(g.chunks, (int)ceil_div((size_t)g.chunks * g.npair, 15)));
    if (g.split > 1) {
        cudaError_t e = op_workspace(op, kWsPart, (size_t)g.split * ep.rows * ep.cols * 4);
        if (e) return e;
        ep.part = (float *)op->ws[kWsPart];
    }
    g.ep = ep;
    cudaError_t e = bn == 64    ? launch_gemm<64, A_MN, B_MN>(op, a, b, g, (unsigned)tiles)
                    : bn == 128 ? launch_gemm<128, A_MN, B_MN>(op, a, b, g, (unsigned)tiles)
                                : launch_gemm<256, A_MN, B_MN>(op, a, b, g, (unsigned)tiles);
    if (!e && g.split > 1) {
        join_splits<<<(unsigned)std::min<size_t>(ceil_div((size_t)ep.rows * ep.cols, 256), (size_t)op->num_sms * 8), 256, 0,
                      op->stream>>>(ep, g.split);
        e = cudaGetLastError();
    }
    return e;
}

int row_ld(int cols) { return (cols + 7) / 8 * 8; }

// An activation or weight tensor as an operand: itself where its rows start on 16 bytes, else a
// copy in the workspace; the three parts of an fp32 one.
cudaError_t as_operand(stacklstm_op *op, const void *src, size_t rows, int cols, int ws, Operand *o)
{
    const int ld = row_ld(cols);
    if (op->dt == SL_BF16 && ld == cols) {
        *o = {src, rows, cols, cols, 1};
        return cudaSuccess;
    }
    const int parts = op->dt == SL_BF16 ? 1 : 3;
    cudaError_t e = op_workspace(op, ws, (size_t)parts * rows * ld * 2);
    if (e) return e;
    const unsigned grid = (unsigned)std::min<size_t>(ceil_div(rows * cols, 256), (size_t)op->num_sms * 16);
    if (op->dt == SL_BF16)
        pack_parts<<<grid, 256, 0, op->stream>>>(rows, cols, ld, (const __nv_bfloat16 *)src, (__nv_bfloat16 *)op->ws[ws]);
    else
        pack_parts<<<grid, 256, 0, op->stream>>>(rows, cols, ld, (const float *)src, (__nv_bfloat16 *)op->ws[ws]);
    *o = {op->ws[ws], rows, cols, ld, parts};
    return cudaGetLastError();
}

}  // namespace
}  // namespace sl

using namespace sl;

extern "C" {

sl_status stacklstm_linear_create(stacklstm_op_t *out, int R, int K, int N, sl_dtype dtype, sl_act act, int device,
                                  void *stream)
{
    if (!out) return SL_ERR_ARG;
    *out = nullptr;
    if (R < 1 || K < 1 || N < 1 || (dtype != SL_FP32 && dtype != SL_BF16) || (int)act < 0 || (int)act >= kActs)
        return SL_ERR_ARG;
    if (K > (1 << 23) || N > (1 << 23) || R > (1 << 28)) return SL_ERR_UNSUPPORTED;
    sl_status st;
    stacklstm_op *op = op_new(SL_OP_LINEAR, dtype, device, stream, &st);
    if (!op) return st;
    op->R = R; op->K = K; op->N = N; op->act = act;
    *out = op;
    return SL_OK;
}

sl_status stacklstm_linear_forward(stacklstm_op_t op, int rows, const void *x, const void *W, const float *bias,
                                   const void *residual, void *y, void *pre)
{
    if (!op || op->kind != SL_OP_LINEAR) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (rows < 0 || rows > op->R) return op_fail(op, SL_ERR_ARG, "rows outside 0 .. R");
    if (rows == 0) return SL_OK;
    if (const char *m = check_pointers({x, W, y}, {bias, residual, pre})) return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    Operand xo, wo;
    cudaError_t e = as_operand(op, x, rows, op->K, kWsX, &xo);
    if (!e) e = as_operand(op, W, op->N, op->K, kWsW, &wo);
    if (!e) {
        Epilogue ep = {};
        ep.rows = rows; ep.cols = op->N; ep.act = op->act; ep.bf16_out = op->dt == SL_BF16;
        ep.bias = bias; ep.residual = residual; ep.y = y; ep.pre = pre;
        e = rows <= 64 ? contract<false, false>(op, wo, xo, op->K, true, ep)
                       : contract<false, false>(op, xo, wo, op->K, false, ep);
    }
    return e ? op_cuda(op, e, "stacklstm_linear_forward") : SL_OK;
}

sl_status stacklstm_linear_backward(stacklstm_op_t op, int rows, const float *dy, const void *x, const void *W,
                                    const void *pre, const float *add, float *dx, float *dW, float *dbias)
{
    if (!op || op->kind != SL_OP_LINEAR) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (rows < 0 || rows > op->R) return op_fail(op, SL_ERR_ARG, "rows outside 0 .. R");
    if (const char *m = check_pointers({}, {dx, dW, dbias})) return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    const int K = op->K, N = op->N;
    cudaError_t e = cudaSuccess;
    if (rows == 0) {  // sums of nothing
        if (dW) e = cudaMemsetAsync(dW, 0, (size_t)N * K * 4, op->stream);
        if (dbias && !e) e = cudaMemsetAsync(dbias, 0, (size_t)N * 4, op->stream);
        return e ? op_cuda(op, e, "stacklstm_linear_backward") : SL_OK;
    }
    if (const char *m = check_pointers({dy}, {pre, add, x, W})) return op_fail(op, SL_ERR_ARG, m);
    if (op->act != kActNone && !pre) return op_fail(op, SL_ERR_ARG, "an activation's backward needs pre");
    if ((dx && !W) || (dW && !x)) return op_fail(op, SL_ERR_ARG, "null pointer");
    // dz in parts, its column sums
    const int ld = row_ld(N);
    const unsigned blocks = ceil_div(rows, kDzRows);
    Operand dz = {nullptr, (size_t)rows, N, ld, 3};
    if (dx || dW) {
        if ((e = op_workspace(op, kWsDz, 3 * (size_t)rows * ld * 2))) return op_cuda(op, e, "stacklstm_linear_backward");
        dz.p = op->ws[kWsDz];
    }
    if (dbias && (e = op_workspace(op, kWsSum, (size_t)blocks * N * 4))) return op_cuda(op, e, "stacklstm_linear_backward");
    const dim3 grid(blocks, ceil_div(N, kDzCols));
    float *sums = dbias ? (float *)op->ws[kWsSum] : nullptr;
    if (op->dt == SL_BF16)
        dz_parts<<<grid, kDzCols, 0, op->stream>>>(rows, N, ld, op->act, dy, (const __nv_bfloat16 *)pre,
                                                   (__nv_bfloat16 *)dz.p, sums);
    else
        dz_parts<<<grid, kDzCols, 0, op->stream>>>(rows, N, ld, op->act, dy, (const float *)pre, (__nv_bfloat16 *)dz.p,
                                                   sums);
    e = cudaGetLastError();
    if (!e && dbias) {
        sum_parts<<<ceil_div(N, 32), 256, 0, op->stream>>>(sums, (int)blocks, N, dbias);
        e = cudaGetLastError();
    }
    if (!e && dx) {
        Operand wo;
        e = as_operand(op, W, N, K, kWsW, &wo);
        Epilogue ep = {};
        ep.rows = rows; ep.cols = K; ep.out = dx; ep.add = add;
        if (!e) e = contract<false, true>(op, dz, wo, N, false, ep);
    }
    if (!e && dW) {
        Operand xo;
        e = as_operand(op, x, rows, K, kWsX, &xo);
        Epilogue ep = {};
        ep.rows = N; ep.cols = K; ep.out = dW;
        if (!e) e = contract<true, true>(op, dz, xo, rows, false, ep);
    }
    return e ? op_cuda(op, e, "stacklstm_linear_backward") : SL_OK;
}

}  // extern "C"
