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

#include <cmath>

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

constexpr int kMaxPairs = 6;

struct GemmArgs {
    int chunks;             // 64-wide chunks of the contraction
    int per_acc;            // chunks to an accumulator
    int split;              // splits of the chunks
    int mt, nt;             // tiles
    int SA, SB;             // ring depths
    int npair, PA, PB;      // partial products; parts of A and of B
    struct Pair {
        uint8_t a, b;       // parts
        uint8_t at_a, at_b; // place of the part among the chunk's loads of A (B)
        uint8_t load_a, load_b, free_a, free_b;  // first (last) use of the part in the chunk
    } pair[kMaxPairs];
    int swapped;            // the output's rows are B's rows (few rows: A = W)
    Epilogue ep;
    long long limit;
    int32_t *err;
};

template <typename T>
__device__ __forceinline__ void finish1(const Epilogue &ep, size_t at, int n, float v)
{
    if (ep.bias) v += ep.bias[n];
    if (ep.pre) ((T *)ep.pre)[at] = from_f32<T>(v);
    v = act_f(v, ep.act);
    if (ep.residual) v += to_f32(((const T *)ep.residual)[at]);
    ((T *)ep.y)[at] = from_f32<T>(v);
}

// One output element.
__device__ __forceinline__ void finish(const Epilogue &ep, int r, int n, float v)
{
    const size_t at = (size_t)r * ep.cols + n;
    if (ep.out)
        ep.out[at] = ep.add ? v + ep.add[at] : v;
    else if (ep.bf16_out)
        finish1<__nv_bfloat16>(ep, at, n, v);
    else
        finish1<float>(ep, at, n, v);
}

// Two neighbours of a row with an even number of columns: accesses of two elements.
__device__ __forceinline__ void finish2(const Epilogue &ep, int r, int n, float2 v, float2 bias)
{
    const size_t at = (size_t)r * ep.cols + n;
    if (ep.out) {
        if (ep.add) {
            const float2 a = *(const float2 *)(ep.add + at);
            v.x += a.x;
            v.y += a.y;
        }
        *(float2 *)(ep.out + at) = v;
        return;
    }
    v.x += bias.x;
    v.y += bias.y;
    float2 o = make_float2(act_f(v.x, ep.act), act_f(v.y, ep.act));
    if (ep.bf16_out) {
        if (ep.pre) *(__nv_bfloat162 *)((__nv_bfloat16 *)ep.pre + at) = __floats2bfloat162_rn(v.x, v.y);
        if (ep.residual) {
            const float2 q = __bfloat1622float2(*(const __nv_bfloat162 *)((const __nv_bfloat16 *)ep.residual + at));
            o.x += q.x;
            o.y += q.y;
        }
        *(__nv_bfloat162 *)((__nv_bfloat16 *)ep.y + at) = __floats2bfloat162_rn(o.x, o.y);
    } else {
        if (ep.pre) *(float2 *)((float *)ep.pre + at) = v;
        if (ep.residual) {
            const float2 q = *(const float2 *)((const float *)ep.residual + at);
            o.x += q.x;
            o.y += q.y;
        }
        *(float2 *)((float *)ep.y + at) = o;
    }
}

constexpr int kEpiWarps = 8;
constexpr int kGemmThreads = (kEpiWarps + 2) * 32;  // then one warp for TMA, one for the MMAs
constexpr int kMaxRing = 16;
constexpr uint32_t kTileA = 128 * 128;  // 128 rows (or 2 x 64 columns) x 64 of the contraction
constexpr uint32_t kStageBytes = kEpiWarps * 32 * 32 * 4;
constexpr uint32_t kRingBytes = 192 * 1024;
constexpr uint32_t kGemmBars = (4 * kMaxRing + 5) * 8 + 16;
constexpr uint32_t kGemmSmem = 1024 + kRingBytes + kStageBytes + kGemmBars;
static_assert(kGemmSmem <= 227 * 1024, "shared memory of a CTA");
constexpr int kGroupM = 16;             // m tiles that share their B tiles in L2
constexpr long long kDrain = 4000000000LL;  // clock cycles: waits for a CTA's own copies and MMAs before it ends

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void *tmap, int c0, int c1, int c2, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"((uint64_t)tmap), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
        : "memory");
}

// D [M][N] += sum over the pairs of A_i B_j^T. A CTA takes units (tile, split) blockIdx.x,
// + gridDim.x, ...; a unit's chunks go through accumulators of per_acc chunks each, two of them
// in turn in tensor memory: warps 0-7 add one up in registers (and after the last finish the
// tile) while the MMAs fill the other. The tensor cores' fp32 additions cut, so an accumulator
// that fp32 results come from takes few of them (1.7e-8 of the result each: 1e-4 after 6012).
// A part is loaded once a chunk, whatever number of products it is in, small products first.
// MN-major operands: blocks of 64 columns, each 64 rows of 128 bytes.
template <int BN, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_parts(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
           const __grid_constant__ GemmArgs g)
{
    constexpr uint32_t kTileB = (uint32_t)BN * 128u;
    constexpr int HALF = BN / 2, SEG = HALF < 32 ? HALF : 32;
    constexpr uint32_t kCols = 2 * BN < 32 ? 32 : 2 * BN;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int SA = g.SA, SB = g.SB;
    const uint32_t ring_a = smem_u32(base), ring_b = ring_a + (uint32_t)SA * kTileA;
    uint64_t *full_a = (uint64_t *)(base + kRingBytes + kStageBytes);
    uint64_t *empty_a = full_a + kMaxRing, *full_b = empty_a + kMaxRing, *empty_b = full_b + kMaxRing;
    uint64_t *acc_full = empty_b + kMaxRing, *acc_empty = acc_full + 2, *done = acc_empty + 2;
    uint32_t *tmem_slot = (uint32_t *)(done + 1);
    volatile int *abort = (volatile int *)(tmem_slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < SA; ++s) {
            tc::mbar_init(&full_a[s], 1);
            tc::mbar_init(&empty_a[s], 1);
        }
        for (int s = 0; s < SB; ++s) {
            tc::mbar_init(&full_b[s], 1);
            tc::mbar_init(&empty_b[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&acc_full[i], 1);
            tc::mbar_init(&acc_empty[i], kEpiWarps);
        }
        tc::mbar_init(done, 1);
        *abort = 0;
        tc::fence_mbar_init();
    }
    if (warp == kEpiWarps) tc::tmem_alloc(tmem_slot, kCols);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto fail = [&]() {
        *abort = 1;
        atomicCAS(g.err, 0, (int)SL_ERR_TIMEOUT);
    };
    const long long limit = g.limit;
    const int tiles = g.mt * g.nt;
    const long long units = (long long)tiles * g.split;
    // unit -> tile and chunks; tiles go down kGroupM m tiles, then to the next n tile, so that the
    // CTAs running at one time share operands in L2
    auto unit = [&](long long u, int &m0, int &n0, int &sp, int &c_lo, int &c_hi) {
        sp = (int)(u / tiles);
        const int t = (int)(u % tiles), group = t / (kGroupM * g.nt), in = t % (kGroupM * g.nt);
        const int first = group * kGroupM, gm = min(kGroupM, g.mt - first);
        m0 = (first + in % gm) * 128;
        n0 = in / gm * BN;
        c_lo = (int)((long long)g.chunks * sp / g.split);
        c_hi = (int)((long long)g.chunks * (sp + 1) / g.split);
    };
    int m0, n0, sp, c_lo, c_hi;

    // a ring's slots in use order: place i of the current chunk, its round's parity
    struct Ring {
        int S, at = 0;
        uint32_t ph = 0;
        __device__ int slot(int i) const { return at + i >= S ? at + i - S : at + i; }
        __device__ uint32_t phase(int i) const { return at + i >= S ? ph ^ 1 : ph; }
        __device__ void next(int parts)
        {
            at += parts;
            if (at >= S) {
                at -= S;
                ph ^= 1;
            }
        }
    };
    Ring ra = {SA}, rb = {SB};

    if (warp == kEpiWarps) {
        if (lane == 0) {
            long long na = 0, nb = 0;  // loads
            bool ok = true;
            for (long long u = blockIdx.x; ok && u < units; u += gridDim.x) {
                unit(u, m0, n0, sp, c_lo, c_hi);
                for (int c = c_lo; ok && c < c_hi; ++c) {
                    const int k0 = c * 64;
                    for (int p = 0; p < g.npair; ++p) {
                        const GemmArgs::Pair &pr = g.pair[p];
                        if (pr.load_b) {
                            const int s = rb.slot(pr.at_b);
                            ok = ok && tc::mbar_wait(&empty_b[s], rb.phase(pr.at_b) ^ 1, limit, abort);
                            if (!ok) break;
                            tc::mbar_arrive_expect_tx(&full_b[s], kTileB);
                            ++nb;
                            const uint32_t dst = ring_b + s * kTileB;
                            if constexpr (B_MN) {
#pragma unroll
                                for (int j = 0; j < BN / 64; ++j)
                                    tma_load_3d(dst + j * 8192, &tm_b, n0 + j * 64, k0, pr.b, &full_b[s]);
                            } else {
                                tma_load_3d(dst, &tm_b, k0, n0, pr.b, &full_b[s]);
                            }
                        }
                        if (pr.load_a) {
                            const int s = ra.slot(pr.at_a);
                            ok = ok && tc::mbar_wait(&empty_a[s], ra.phase(pr.at_a) ^ 1, limit, abort);
                            if (!ok) break;
                            tc::mbar_arrive_expect_tx(&full_a[s], kTileA);
                            ++na;
                            const uint32_t dst = ring_a + s * kTileA;
                            if constexpr (A_MN) {
                                tma_load_3d(dst, &tm_a, m0, k0, pr.a, &full_a[s]);
                                tma_load_3d(dst + 8192, &tm_a, m0 + 64, k0, pr.a, &full_a[s]);
                            } else {
                                tma_load_3d(dst, &tm_a, k0, m0, pr.a, &full_a[s]);
                            }
                        }
                    }
                    ra.next(g.PA);
                    rb.next(g.PB);
                }
            }
            if (!ok) fail();
            // no copy in flight when the CTA ends: the last load of every slot has landed
            for (int s = 0; s < SA; ++s)
                if (na > s) tc::mbar_wait(&full_a[s], (uint32_t)((na - 1 - s) / SA) & 1, kDrain, nullptr);
            for (int s = 0; s < SB; ++s)
                if (nb > s) tc::mbar_wait(&full_b[s], (uint32_t)((nb - 1 - s) / SB) & 1, kDrain, nullptr);
        }
        __syncwarp();
    } else if (warp == kEpiWarps + 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = tc::idesc_bf16(BN, A_MN, B_MN);
            uint32_t acc = 0;  // accumulators filled so far
            bool ok = true;
            for (long long u = blockIdx.x; ok && u < units; u += gridDim.x) {
                unit(u, m0, n0, sp, c_lo, c_hi);
                for (int c = c_lo; ok && c < c_hi; ++acc) {
                    const uint32_t d = tmem + (acc & 1) * BN;
                    ok = tc::mbar_wait(&acc_empty[acc & 1], ((acc >> 1) & 1) ^ 1, limit, abort);
                    if (!ok) break;
                    tc::tc_fence_after();
                    const int c_end = min(c_hi, c + g.per_acc);
                    uint32_t more = 0;
                    for (; ok && c < c_end; ++c) {
                        for (int p = 0; p < g.npair; ++p) {
                            const GemmArgs::Pair &pr = g.pair[p];
                            const int sa = ra.slot(pr.at_a), sb = rb.slot(pr.at_b);
                            if (pr.load_b) ok = tc::mbar_wait(&full_b[sb], rb.phase(pr.at_b), limit, abort);
                            if (ok && pr.load_a) ok = tc::mbar_wait(&full_a[sa], ra.phase(pr.at_a), limit, abort);
                            if (!ok) break;
                            tc::tc_fence_after();
                            const uint32_t as = ring_a + sa * kTileA, bs = ring_b + sb * kTileB;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {  // 16 of the contraction: 32 bytes of a row, or 16 rows
                                tc::mma_bf16(d, A_MN ? tc::smem_desc(as + k * 2048, 8192, 1024) : tc::smem_desc(as + k * 32, 16, 1024),
                                             B_MN ? tc::smem_desc(bs + k * 2048, 8192, 1024) : tc::smem_desc(bs + k * 32, 16, 1024),
                                             idesc, more);
                                more = 1;
                            }
                            if (pr.free_a) tc::mma_commit(&empty_a[sa]);
                            if (pr.free_b) tc::mma_commit(&empty_b[sb]);
                        }
                        ra.next(g.PA);
                        rb.next(g.PB);
                    }
                    if (ok) tc::mma_commit(&acc_full[acc & 1]);
                }
            }
            if (!ok) fail();
            tc::mma_commit(done);
            tc::mbar_wait(done, 0, kDrain, nullptr);  // no MMA in flight when tensor memory is freed
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------ sums and outputs
        const int q = warp & 3, half = warp >> 2;  // a warp reads its quadrant of the lanes
        float *stage = (float *)(base + kRingBytes) + warp * 1024;
        const Epilogue &ep = g.ep;
        uint32_t acc = 0;
        bool ok = true;
        for (long long u = blockIdx.x; ok && u < units; u += gridDim.x) {
            unit(u, m0, n0, sp, c_lo, c_hi);
            float sum[HALF];
            for (int c = c_lo; c < c_hi; c += g.per_acc, ++acc) {
                // (the whole warp: its reads of tensor memory are collective)
                ok = __all_sync(0xffffffffu, tc::mbar_wait(&acc_full[acc & 1], (acc >> 1) & 1, limit, abort));
                if (!ok) break;
                tc::tc_fence_after();
                const uint32_t at = tmem + ((uint32_t)(q * 32) << 16) + (acc & 1) * BN + half * HALF;
                if (c == c_lo) {
#pragma unroll
                    for (int i = 0; i < HALF; i += 16) tc::tmem_ld16(at + i, *(float(*)[16])(sum + i));
                } else {
#pragma unroll
                    for (int i = 0; i < HALF; i += 16) {
                        float v[16];
                        tc::tmem_ld16(at + i, v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[i + j] += v[j];
                    }
                }
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&acc_empty[acc & 1]);
            }
            if (!ok) break;
            // through shared memory, 32 rows x SEG columns at a time (16-byte pieces of row r at
            // piece ^ (r mod 8)), so that a row's neighbours are a warp's
            const int mm = m0 + q * 32, nn = n0 + half * HALF;
            Epilogue o = ep;
            if (ep.part) {  // plain sums
                o.out = ep.part + (size_t)sp * ep.rows * ep.cols;
                o.add = nullptr;
            }
            const bool pairs = ep.cols % 2 == 0;
#pragma unroll
            for (int s0 = 0; s0 < HALF; s0 += SEG) {
#pragma unroll
                for (int i = 0; i < SEG / 4; ++i)
                    *(float4 *)(stage + lane * 32 + ((i ^ (lane & 7)) << 2)) =
                        make_float4(sum[s0 + 4 * i], sum[s0 + 4 * i + 1], sum[s0 + 4 * i + 2], sum[s0 + 4 * i + 3]);
                __syncwarp();
                if (g.swapped) {
                    const int n = mm + lane;
                    for (int i = 0; i < SEG; ++i) {
                        const int r = nn + s0 + i;
                        if (n < ep.cols && r < ep.rows) finish(o, r, n, stage[lane * 32 + (((i >> 2) ^ (lane & 7)) << 2) + (i & 3)]);
                    }
                } else if (pairs && SEG == 32) {
                    const int j = lane & 15, n = nn + s0 + 2 * j;
                    float2 bias = make_float2(0.0f, 0.0f);
                    if (n < ep.cols && !o.out && ep.bias) bias = *(const float2 *)(ep.bias + n);
                    if (n < ep.cols)
#pragma unroll 4
                        for (int i = 0; i < 16; ++i) {
                            const int rr = 2 * i + (lane >> 4), r = mm + rr;
                            if (r < ep.rows)
                                finish2(o, r, n, *(const float2 *)(stage + rr * 32 + (((j >> 1) ^ (rr & 7)) << 2) + ((j & 1) << 1)), bias);
                        }
                } else {
                    const int j = lane, n = nn + s0 + j;
                    if (j < SEG && n < ep.cols)
                        for (int rr = 0; rr < 32; ++rr)
                            if (mm + rr < ep.rows) finish(o, mm + rr, n, stage[rr * 32 + (((j >> 2) ^ (rr & 7)) << 2) + (j & 3)]);
                }
                __syncwarp();
            }
        }
        if (!ok && lane == 0) fail();
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == kEpiWarps) tc::tmem_dealloc(tmem, kCols);
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
cudaError_t launch_gemm(const stacklstm_op *op, const Operand &a, const Operand &b, const GemmArgs &g)
{
    CUtensorMap ta, tb;
    cudaError_t e = operand_map(&ta, a, A_MN ? 64 : 128);
    if (!e) e = operand_map(&tb, b, B_MN ? 64 : BN);
    if (!e) e = smem_at_least((const void *)gemm_parts<BN, A_MN, B_MN>, kGemmSmem);
    if (e) return e;
    const unsigned grid = (unsigned)std::min<long long>((long long)g.mt * g.nt * g.split, op->num_sms);
    gemm_parts<BN, A_MN, B_MN><<<grid, kGemmThreads, kGemmSmem, op->stream>>>(ta, tb, g);
    return cudaGetLastError();
}

enum { kWsX = 0, kWsW, kWsDz, kWsSum, kWsPart };  // workspace buffers

constexpr size_t kMostPartBytes = (size_t)1 << 30;  // of the splits' sums

// Tile width and splits: the least of waves x chunks x cycles a chunk (two cycles a column and
// product, and no fewer than the operands' bytes take at 64 a cycle), a tile's start and end, and
// for a split contraction its sums written and read again, and a second launch.
void plan_gemm(GemmArgs &g, int M, int N, int bn_lo, int bn_hi, size_t out_elems, int sms, int *bn_out)
{
    double best = 1e300;
    for (int bn = bn_lo; bn <= bn_hi; bn *= 2) {
        const double mt = ceil_div(M, 128), nt = ceil_div(N, bn);
        const double cyc = std::max(2.0 * bn * g.npair, (g.PA * (double)kTileA + g.PB * bn * 128.0) / 64.0);
        for (int split = 1; split <= std::min(g.chunks, 64); ++split) {
            if (split > 1 && (g.chunks / split < 2 || (double)split * out_elems * 4 > (double)kMostPartBytes)) break;
            const double waves = std::ceil(mt * nt * split / sms), chunks = std::ceil((double)g.chunks / split);
            double cost = waves * (chunks * cyc + 400.0) + 16.0 * bn + 2000.0;
            if (split > 1) cost += 5000.0 + 2.0 * split * out_elems * 4 / 3500.0;
            if (cost < best) {
                best = cost;
                g.mt = (int)mt;
                g.nt = (int)nt;
                g.split = split;
                *bn_out = bn;
            }
        }
    }
}

// D = sum over the parts' products of A B^T, kcols long, and its epilogue.
template <bool A_MN, bool B_MN>
cudaError_t contract(stacklstm_op *op, const Operand &a, const Operand &b, int kcols, bool swapped, Epilogue ep)
{
    GemmArgs g = {};
    g.chunks = (int)ceil_div(kcols, 64);
    g.PA = a.parts;
    g.PB = b.parts;
    // partial products, small ones first; a part's place is that of its first use
    int next_a = 0, next_b = 0, place_a[3] = {-1, -1, -1}, place_b[3] = {-1, -1, -1};
    for (int order = 2; order >= 0; --order)
        for (int i = 0; i < a.parts; ++i) {
            const int j = order - i;
            if (j < 0 || j >= b.parts) continue;
            GemmArgs::Pair &p = g.pair[g.npair++];
            p.a = (uint8_t)i;
            p.b = (uint8_t)j;
            if ((p.load_a = place_a[i] < 0)) place_a[i] = next_a++;
            if ((p.load_b = place_b[j] < 0)) place_b[j] = next_b++;
            p.at_a = (uint8_t)place_a[i];
            p.at_b = (uint8_t)place_b[j];
        }
    for (int i = 0; i < a.parts; ++i)
        for (int p = g.npair - 1; p >= 0; --p)
            if (g.pair[p].a == i) {
                g.pair[p].free_a = 1;
                break;
            }
    for (int j = 0; j < b.parts; ++j)
        for (int p = g.npair - 1; p >= 0; --p)
            if (g.pair[p].b == j) {
                g.pair[p].free_b = 1;
                break;
            }
    // fp32 results: 24 MMAs to an accumulator
    g.per_acc = ep.out || !ep.bf16_out ? std::max(1, 6 / g.npair) : g.chunks;
    g.swapped = swapped;
    g.limit = op->wait_limit;
    g.err = op->err;
    const int M = swapped ? ep.cols : ep.rows, N = swapped ? ep.rows : ep.cols;
    // (three parts of a 256-wide B leave the rings no second chunk)
    const int most = b.parts == 3 ? 128 : 256;
    const int lo = swapped && N <= 32 ? 32 : 64, hi = N <= lo ? lo : N <= 64 ? 64 : N <= 128 ? 128 : most;
    int bn = 64;
    plan_gemm(g, M, N, lo, hi, (size_t)ep.rows * ep.cols, op->num_sms, &bn);
    // rings: as many whole chunks as fit, what is left to B, then to A
    const uint32_t tb = (uint32_t)bn * 128, per = g.PA * kTileA + g.PB * tb;
    const int depth = (int)(kRingBytes / per);
    g.SA = std::min(kMaxRing / g.PA, depth) * g.PA;
    g.SB = std::min(kMaxRing / g.PB, depth) * g.PB;
    while (g.SB < kMaxRing && g.SA * kTileA + (g.SB + 1) * tb <= kRingBytes && g.PB < g.PA) ++g.SB;
    while (g.SA < kMaxRing && (g.SA + 1) * kTileA + g.SB * tb <= kRingBytes) ++g.SA;
    if (g.split > 1) {
        cudaError_t e = op_workspace(op, kWsPart, (size_t)g.split * ep.rows * ep.cols * 4);
        if (e) return e;
        ep.part = (float *)op->ws[kWsPart];
    }
    g.ep = ep;
    cudaError_t e = cudaErrorInvalidValue;
    if constexpr (!A_MN && !B_MN)
        if (bn == 32) e = launch_gemm<32, A_MN, B_MN>(op, a, b, g);
    if (bn == 64) e = launch_gemm<64, A_MN, B_MN>(op, a, b, g);
    if (bn == 128) e = launch_gemm<128, A_MN, B_MN>(op, a, b, g);
    if (bn == 256) e = launch_gemm<256, A_MN, B_MN>(op, a, b, g);
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
