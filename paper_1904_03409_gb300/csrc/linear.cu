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
// dz is written once, as three bf16 parts, with the column sums of dbias, in the launch that also
// makes the parts of an fp32 x and W.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <cmath>
#include <type_traits>

#include "op.cuh"
#include "tc.cuh"

namespace sl {
namespace {

using tc::smem_u32;

enum { kActNone = 0, kActRelu, kActTanh, kActGelu, kActSilu, kActs };

__device__ __forceinline__ float rcp_hw(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float exp2_hw(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
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
// The same for a result that is rounded to bf16. Phi(z) = 1 - h / 2 (z >= 0), h / 2 (z < 0) with
// h = erfc(|z| / sqrt 2) = t (a1 + t (a2 + ...)) exp(-z^2 / 2), t = 1 / (1 + p |z| / sqrt 2), by formula
// 7.1.26 of Abramowitz and Stegun's Handbook of Mathematical Functions (of erf, error 1.5e-7: of gelu
// 2e-7 in all, below bf16 rounding down to z = -5; relative to what is left of it there, 2e-3 at -5,
// 2e-2 at -10), a third of erff's instructions, which bounded the layer; the sigmoid by the hardware's
// exponential and quotient (2^-21; the quotient is 0 below z = -87.3, where silu is above -1.1e-36).
__device__ __forceinline__ float act_f_bf16(float z, int act)
{
    if (act == kActGelu) {
        const float x = fabsf(z) * 0.70710678f;
        const float t = rcp_hw(fmaf(0.3275911f, x, 1.0f));
        float h = fmaf(t, 1.061405429f, -1.453152027f);
        h = fmaf(t, h, 1.421413741f);
        h = fmaf(t, h, -0.284496736f);
        h = fmaf(t, h, 0.254829592f);
        h *= t * exp2_hw(x * x * -1.44269504f);
        return fmaf(-0.5f * fminf(fabsf(z), 64.0f), h, fmaxf(z, 0.0f));  // (z - z h / 2, -|z| h / 2; no inf x 0)
    }
    if (act == kActSilu) return __fdividef(z, 1.0f + __expf(-z));
    return act_f(z, act);
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

// What a call makes of its tensors before the contractions, in one launch: x and W as parts (or, bf16
// whose rows do not start on 16 bytes, as a copy whose rows do), and dz = dy act'(pre) as parts with
// its column sums. Each is a range of CTAs.
struct Pack {
    const void *src;        // [rows][cols], or null
    __nv_bfloat16 *out;     // [parts][rows][ld]
    size_t rows;
    int cols, ld;
    unsigned ctas;
};
struct Dz {
    const float *dy;
    const void *pre;
    __nv_bfloat16 *out;     // [3][rows][ld], or null
    float *part;            // [row blocks][N] column sums, or null
    float *dbias;
    int *arrived;           // [column blocks], 0 between calls
    int rows, N, ld, act;
    int lanes;              // of a warp to a row: 32, or as few (a power of 2) as four columns each fill
    unsigned row_blocks, ctas;
};
struct Prepare {
    Pack x, w;
    Dz dz;
};

constexpr int kPackItems = 4;  // groups of four columns a thread
constexpr int kDzCols = 128, kDzRows = 64, kDzSub = 8;  // a block's columns at most, its rows, its warps

// Groups of four columns, 8 bytes a part. (The groups of `out` follow one another whatever the rows'
// length is; those of src do where its rows are as long.)
template <typename T>
__device__ __forceinline__ void pack_block(const Pack &a, unsigned cta)
{
    const size_t per = (size_t)a.ld / 4, groups = a.rows * per, plane = a.rows * a.ld;
    const bool flat = a.cols == a.ld, quads = a.cols % 4 == 0;
    const T *src = (const T *)a.src;
    float v[kPackItems][4];
    T raw[kPackItems][4];
#pragma unroll
    for (int u = 0; u < kPackItems; ++u) {
        const size_t g = (size_t)cta * (256 * kPackItems) + u * 256 + threadIdx.x;
        if (g >= groups) break;
        const size_t r = flat ? 0 : g / per;
        const int c = flat ? 0 : (int)(g - r * per) * 4;
        const T *p = flat ? src + g * 4 : src + r * a.cols + c;
        const int n = flat ? 4 : a.cols - c;  // columns left (the last groups of a row may be past them)
        if constexpr (sizeof(T) == 4) {
            if (quads && n >= 4) {
                const float4 q = *(const float4 *)p;
                v[u][0] = q.x; v[u][1] = q.y; v[u][2] = q.z; v[u][3] = q.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[u][j] = j < n ? p[j] : 0.0f;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) raw[u][j] = j < n ? p[j] : from_f32<T>(0.0f);
        }
    }
#pragma unroll
    for (int u = 0; u < kPackItems; ++u) {
        const size_t g = (size_t)cta * (256 * kPackItems) + u * 256 + threadIdx.x;
        if (g >= groups) break;
        union {
            __nv_bfloat16 b[4];
            uint2 q;
        } o[3];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                __nv_bfloat16 p[3];
                split3(v[u][j], p);
#pragma unroll
                for (int k = 0; k < 3; ++k) o[k].b[j] = p[k];
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) *(uint2 *)(a.out + k * plane + g * 4) = o[k].q;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) o[0].b[j] = raw[u][j];
            *(uint2 *)(a.out + g * 4) = o[0].q;
        }
    }
}

// dz of kDzRows rows and up to kDzCols columns, and the column sums of it. A lane takes four columns
// (one 8-byte store a part, from one 16-byte read where the rows of dy start on 16 bytes), a.lanes of
// them a row (a warp several rows of a narrow layer), four rows at a time; the threads' sums of a
// column are added in order, and so are, by the last block of a column block to end, the blocks'.
// HBM-bound: 4 + 6 bytes an element.
template <typename T, int LANES>  // (0: a.lanes)
__device__ __forceinline__ void dz_block(const Dz &a, unsigned cta)
{
    __shared__ float4 sm[32 * kDzSub];
    __shared__ int last;
    const int lanes = LANES ? LANES : a.lanes;
    const int N = a.N, lane = threadIdx.x % lanes, sub = threadIdx.x / lanes, subs = 32 * kDzSub / lanes;
    const unsigned rb = cta % a.row_blocks, cb = cta / a.row_blocks;
    const int c = (int)cb * kDzCols + lane * 4, nc = min(4, N - c);
    const int r0 = (int)rb * kDzRows, r1 = min(a.rows, r0 + kDzRows);
    const size_t plane = (size_t)a.rows * a.ld;
    const bool quads = N % 4 == 0;
    const T *pre = (const T *)a.pre;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (nc > 0) {
        for (int r = r0 + sub; r < r1; r += 4 * subs) {
            float v[4][4], z[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ri = r + i * subs;
                const size_t at = (size_t)ri * N + c;
                if (quads) {
                    const float4 q = ri < r1 ? *(const float4 *)(a.dy + at) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    v[i][0] = q.x; v[i][1] = q.y; v[i][2] = q.z; v[i][3] = q.w;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i][j] = ri < r1 && j < nc ? a.dy[at + j] : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) z[i][j] = a.act != kActNone && ri < r1 && j < nc ? to_f32(pre[at + j]) : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ri = r + i * subs;
                if (ri >= r1) break;
                union {
                    __nv_bfloat16 b[4];
                    uint2 q;
                } o[3];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float w = a.act != kActNone ? __fmul_rn(v[i][j], act_grad(z[i][j], a.act)) : v[i][j];  // (not fused with the sum)
                    sum[j] += w;
                    __nv_bfloat16 p[3];
                    split3(w, p);
#pragma unroll
                    for (int k = 0; k < 3; ++k) o[k].b[j] = p[k];
                }
                if (a.out)  // (a row has room for whole groups of eight: what is past N is never read)
#pragma unroll
                    for (int k = 0; k < 3; ++k) *(uint2 *)(a.out + k * plane + (size_t)ri * a.ld + c) = o[k].q;
            }
        }
    }
    if (!a.part) return;
    // the threads' sums of each column in order, to the first `lanes` threads
    auto joined = [&](const float4 &mine) {
        sm[threadIdx.x] = mine;
        __syncthreads();
        float4 t = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (sub == 0)
#pragma unroll 8
            for (int i = 0; i < subs; ++i) {
                const float4 q = sm[i * lanes + lane];
                t.x += q.x; t.y += q.y; t.z += q.z; t.w += q.w;
            }
        return t;
    };
    auto put = [&](float *to, const float4 &t) {
        const float w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < nc) to[j] = w[j];
    };
    float4 t = joined(make_float4(sum[0], sum[1], sum[2], sum[3]));
    if (sub == 0) {
        put(a.part + (size_t)rb * N + c, t);
        __threadfence();
    }
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(&a.arrived[cb], 1) == (int)a.row_blocks - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (threadIdx.x == 0) a.arrived[cb] = 0;  // for the next call
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (unsigned s = sub; s < a.row_blocks; s += subs)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < nc) acc[j] += __ldcg(a.part + (size_t)s * N + c + j);
    t = joined(make_float4(acc[0], acc[1], acc[2], acc[3]));
    if (sub == 0) put(a.dbias + c, t);
}

// Bound by HBM: dz of 4096 x 32003 is read as 4 bytes and written as 6 in 245 us (5.4 TB/s).
template <typename T>
__global__ void __launch_bounds__(256)
prepare(const __grid_constant__ Prepare a)
{
    after_previous();
    unsigned cta = blockIdx.x;
    if (cta < a.dz.ctas) return a.dz.lanes == 32 ? dz_block<T, 32>(a.dz, cta) : dz_block<T, 0>(a.dz, cta);
    cta -= a.dz.ctas;
    if (cta < a.x.ctas) return pack_block<T>(a.x, cta);
    pack_block<T>(a.w, cta - a.x.ctas);
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
    int per_acc;            // chunks to an accumulator
    int split;              // splits of the chunks
    int K, N;               // of the contraction, and rows of B
    int mt, nt, step;       // tiles, and rows of B from one to the next (fp32 results: as few as nt allows)
    int SA, SB;             // ring depths
    int swapped;            // the output's rows are B's rows (few rows: A = W)
    Epilogue ep;
    long long limit;
    int32_t *err;
};

// The partial products of PA parts of A and PB of B: those of order i + j <= 2, small ones first.
template <int PA, int PB>
struct Pairs {
    int n = 0, a[6] = {}, b[6] = {};
    int at_a[3] = {}, at_b[3] = {};      // place of a part among the chunk's loads: that of its first use
    bool load_a[6] = {}, load_b[6] = {}, free_a[6] = {}, free_b[6] = {};
    constexpr Pairs()
    {
        int na = 0, nb = 0;
        bool seen_a[3] = {}, seen_b[3] = {};
        for (int order = 2; order >= 0; --order)
            for (int i = 0; i < PA; ++i) {
                const int j = order - i;
                if (j < 0 || j >= PB) continue;
                a[n] = i;
                b[n] = j;
                load_a[n] = !seen_a[i];
                load_b[n] = !seen_b[j];
                if (!seen_a[i]) at_a[i] = na++;
                if (!seen_b[j]) at_b[j] = nb++;
                seen_a[i] = seen_b[j] = true;
                ++n;
            }
        for (int p = 0; p < n; ++p) {
            free_a[p] = free_b[p] = true;
            for (int q = p + 1; q < n; ++q) {
                if (a[q] == a[p]) free_a[p] = false;
                if (b[q] == b[p]) free_b[p] = false;
            }
        }
    }
};

// What an output is made of, with the pointers of its kind: plain fp32 sums (and an addend), or
// the forward's y and pre of type T.
template <typename T>
struct Forward {
    const T *residual;
    T *y, *pre;
    int act;
    __device__ explicit Forward(const Epilogue &ep) : residual((const T *)ep.residual), y((T *)ep.y), pre((T *)ep.pre), act(ep.act) {}
    __device__ __forceinline__ float extra(size_t at) const { return residual ? to_f32(residual[at]) : 0.0f; }
    __device__ __forceinline__ void put(size_t at, float v, float bias, float extra) const
    {
        v += bias;
        if (pre) pre[at] = from_f32<T>(v);
        y[at] = from_f32<T>((sizeof(T) == 2 ? act_f_bf16(v, act) : act_f(v, act)) + extra);
    }
};
struct Plain {
    const float *add;
    float *out;
    __device__ __forceinline__ float extra(size_t at) const { return add ? add[at] : 0.0f; }
    __device__ __forceinline__ void put(size_t at, float v, float, float extra) const { out[at] = v + extra; }
};

// Four neighbours in one access.
constexpr int kFew = 4;
__device__ __forceinline__ void store_few(float *p, const float (&v)[kFew]) { *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store_few(__nv_bfloat16 *p, const float (&v)[kFew])
{
    union {
        __nv_bfloat162 b[2];
        uint2 q;
    } o;
    o.b[0] = __floats2bfloat162_rn(v[0], v[1]);
    o.b[1] = __floats2bfloat162_rn(v[2], v[3]);
    *(uint2 *)p = o.q;
}
// The same as it lies in memory, and its values.
template <typename T>
struct Few {
    using Q = typename std::conditional<sizeof(T) == 4, float4, uint2>::type;
    Q q;
    __device__ __forceinline__ void load(const T *p) { q = *(const Q *)p; }
    __device__ __forceinline__ float get(int i) const { return to_f32(((const T *)&q)[i]); }
};

// A warp's 32 rows x SEG columns of sums in shared memory: row r's 16-byte pieces at piece ^ (r mod 8).
__device__ __forceinline__ const float *staged(const float *stage, int r, int c)
{
    return stage + r * 32 + (((c >> 2) ^ (r & 7)) << 2) + (c & 3);
}

// Those sums (row 0 = output row r0, column 0 = output column n0) to an output of any number of
// columns, a row's neighbours by neighbouring lanes; what is added is read eight rows ahead of the
// stores.
template <int SEG, typename T, bool FORWARD, int ACT>
__device__ __forceinline__ void put_rows(const float *stage, int lane, int r0, int n0, int n_end, int rows, int cols,
                                         const float *bias_p, const T *extra_p, T *y, T *pre)
{
    const int n = n0 + lane;
    if (lane >= SEG || n >= n_end) return;
    const float bias = FORWARD && bias_p ? bias_p[n] : 0.0f;
    const int m = min(32, rows - r0);
    size_t at = (size_t)r0 * cols + n;
#pragma unroll 1
    for (int i0 = 0; i0 < m; i0 += 8, at += 8 * (size_t)cols) {
        float extra[8] = {};
        if (extra_p)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i0 + i < m) extra[i] = to_f32(extra_p[at + i * (size_t)cols]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i0 + i < m) {
                float v = *staged(stage, i0 + i, lane) + bias;
                if (FORWARD) {
                    if (pre) pre[at + i * (size_t)cols] = from_f32<T>(v);
                    v = sizeof(T) == 2 ? act_f_bf16(v, ACT) : act_f(v, ACT);
                }
                y[at + i * (size_t)cols] = from_f32<T>(v + extra[i]);
            }
    }
}
template <int SEG, typename T>
__device__ __forceinline__ void put_rows_forward(const Epilogue &ep, const float *stage, int lane, int r0, int n0, int n_end)
{
    const T *res = (const T *)ep.residual;
    T *y = (T *)ep.y, *pre = (T *)ep.pre;
    switch (ep.act) {
    case kActRelu: return put_rows<SEG, T, true, kActRelu>(stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    case kActTanh: return put_rows<SEG, T, true, kActTanh>(stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    case kActGelu: return put_rows<SEG, T, true, kActGelu>(stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    case kActSilu: return put_rows<SEG, T, true, kActSilu>(stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    default: return put_rows<SEG, T, true, kActNone>(stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    }
}

// The same of an output that is D's transpose: stage row i is output column n0 + i.
template <int SEG, typename Out>
__device__ __forceinline__ void put_cols(const Out &o, const float *stage, int lane, int r0, int r_end, int n0, int cols,
                                         const float *bias_p)
{
    const int n = n0 + lane;
    if (n >= cols) return;
    const float bias = bias_p ? bias_p[n] : 0.0f;
    const int m = min(SEG, r_end - r0);
    for (int i0 = 0; i0 < m; i0 += 4) {
        float extra[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) extra[i] = i0 + i < m ? o.extra((size_t)(r0 + i0 + i) * cols + n) : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i0 + i < m) o.put((size_t)(r0 + i0 + i) * cols + n, *staged(stage, lane, i0 + i), bias, extra[i]);
    }
}

// A warp's 32 rows x 32 NSEG columns of an output whose number of columns 4 divides (n_end too): four
// neighbours a lane, four rows at a time; stage_in(seg) brings 32 columns of sums into `stage` (false: a
// wait ran out). What is added to a block of 32 columns (residual, add) is read while the block
// before it is worked on, the first one's while the sums are waited for, and rows are finished a few
// at a time (more of them keep more activations in flight than there are registers).
template <typename T, bool FORWARD, int ACT, int NSEG, typename StageIn>
__device__ __forceinline__ bool put_few(const StageIn &stage_in, const float *stage, int lane, int r0, int n0, int n_end, int rows, int cols,
                                        const float *bias_p, const T *extra_p, T *y, T *pre)
{
    constexpr int W = kFew, L = 32 / W, NI = 32 / W;  // lanes a row; steps of W rows
    const int j = lane % L * W, sub = lane / L, m = min(32, rows - r0);
    const size_t step = W * (size_t)cols, first = (size_t)(r0 + sub) * cols + n0 + j;
    Few<T> next[NI] = {}, extra[NI];
    auto fetch = [&](int seg) {
        if (n0 + seg * 32 + j < n_end)
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (sub + W * i < m) next[i].load(extra_p + first + seg * 32 + i * step);
    };
    if (extra_p) fetch(0);
#pragma unroll 1
    for (int seg = 0; seg < NSEG; ++seg) {
        if (!stage_in(seg)) return false;
#pragma unroll
        for (int i = 0; i < NI; ++i) extra[i] = next[i];
        if (extra_p && seg + 1 < NSEG) fetch(seg + 1);
        const int n = n0 + seg * 32 + j;
        float bias[W] = {};
        if (FORWARD && bias_p && n < n_end)
#pragma unroll
            for (int k = 0; k < W; ++k) bias[k] = bias_p[n + k];
        __syncwarp();
        if (n < n_end) {
            const size_t at = first + seg * 32;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                if (sub + W * i < m) {
                    Few<float> s;
                    s.load(staged(stage, sub + W * i, j));
                    float v[W];
#pragma unroll
                    for (int k = 0; k < W; ++k) v[k] = s.get(k) + (FORWARD ? bias[k] : 0.0f);
                    if (FORWARD && pre) store_few(pre + at + i * step, v);
#pragma unroll
                    for (int k = 0; k < W; ++k) {
                        if (FORWARD) v[k] = sizeof(T) == 2 ? act_f_bf16(v[k], ACT) : act_f(v[k], ACT);
                        v[k] += extra[i].get(k);
                    }
                    store_few(y + at + i * step, v);
                }
                if (i % (8 / W) == 8 / W - 1) asm volatile("" ::: "memory");
            }
        }
        __syncwarp();
    }
    return true;
}
template <typename T, int NSEG, typename StageIn>
__device__ __forceinline__ bool put_forward(const StageIn &in, const Epilogue &ep, const float *stage, int lane, int r0, int n0, int n_end)
{
    const T *res = (const T *)ep.residual;
    T *y = (T *)ep.y, *pre = (T *)ep.pre;
    switch (ep.act) {
    case kActRelu: return put_few<T, true, kActRelu, NSEG>(in, stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    case kActTanh: return put_few<T, true, kActTanh, NSEG>(in, stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    case kActGelu: return put_few<T, true, kActGelu, NSEG>(in, stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    case kActSilu: return put_few<T, true, kActSilu, NSEG>(in, stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    default: return put_few<T, true, kActNone, NSEG>(in, stage, lane, r0, n0, n_end, ep.rows, ep.cols, ep.bias, res, y, pre);
    }
}

// A warp's 32 rows x SEG NSEG columns of sums to the output, those of D's columns before n_end
// (FIT) or all of its columns.
template <int SEG, int NSEG, bool GRADIENT, bool FIT, typename StageIn>
__device__ __forceinline__ bool put_tile(const StageIn &in, const Epilogue &ep, bool swapped, int sp, const float *stage,
                                         int lane, int m0, int n0, int n_end)
{
    const int c_end = FIT ? n_end : ep.cols, r_end = FIT ? n_end : ep.rows;  // (D's columns are the output's, or, swapped, its rows)
    const bool plain = GRADIENT || ep.part;
    const Plain p = {ep.part ? nullptr : ep.add, ep.part ? ep.part + (size_t)sp * ep.rows * ep.cols : ep.out};
    if (SEG == 32 && ep.cols % 4 == 0 && (GRADIENT || !swapped)) {
        if (plain)
            return put_few<float, false, kActNone, NSEG>(in, stage, lane, m0, n0, c_end, ep.rows, ep.cols, nullptr, p.add, p.out, nullptr);
        if constexpr (!GRADIENT)
            return ep.bf16_out ? put_forward<__nv_bfloat16, NSEG>(in, ep, stage, lane, m0, n0, c_end)
                               : put_forward<float, NSEG>(in, ep, stage, lane, m0, n0, c_end);
    }
#pragma unroll 1
    for (int seg = 0; seg < NSEG; ++seg, n0 += SEG) {
        if (!in(seg)) return false;
        __syncwarp();
        if (!GRADIENT && swapped) {
            if (plain)
                put_cols<SEG>(p, stage, lane, n0, r_end, m0, ep.cols, nullptr);
            else if (ep.bf16_out)
                put_cols<SEG>(Forward<__nv_bfloat16>(ep), stage, lane, n0, r_end, m0, ep.cols, ep.bias);
            else
                put_cols<SEG>(Forward<float>(ep), stage, lane, n0, r_end, m0, ep.cols, ep.bias);
        } else {
            if (plain)
                put_rows<SEG, float, false, kActNone>(stage, lane, m0, n0, c_end, ep.rows, ep.cols, nullptr, p.add, p.out, nullptr);
            else if constexpr (!GRADIENT) {
                if (ep.bf16_out)
                    put_rows_forward<SEG, __nv_bfloat16>(ep, stage, lane, m0, n0, c_end);
                else
                    put_rows_forward<SEG, float>(ep, stage, lane, m0, n0, c_end);
            }
        }
        __syncwarp();
    }
    return true;
}

// Warp 0 for TMA, warp 1 for the MMAs (2 and 3 idle), then the warps for the sums and outputs: eight
// where they add accumulators up (launched with 168 registers a thread, 384 x 168 = 64512, of which
// the first group keeps 56 and the others take 224, 128 x 56 + 256 x 224 = 64512, so that 128 sums
// and a batch of reads stay in registers), else sixteen, whose activations hide one another's
// latencies (96 registers a thread, 640 x 96 = 61440, split as 128 x 32 + 512 x 112 = 61440).
// A bf16 forward of up to 32 rows reads W and does little else: two CTAs an SM with half the shared
// memory and four output warps each, so that one's start and outputs, and the next launch's start,
// lie under the other's loads. 8 rows, K = 1024, N = 600: 5.9 us so, 7.3 with one CTA of eight output
// warps; N = 32003 14.9 and 16.4, of 32 rows 18.1 and 17.5; N = 9728, whose 76 tiles then have half
// an SM's loads in flight each, 9.7 and 9.1. Up to 64 rows 23.9 and 20.6: one CTA.
constexpr int gemm_ctas(int bn, bool sums) { return !sums && bn == 32 ? 2 : 1; }
constexpr int gemm_epi_warps(int bn, bool sums) { return !sums && bn >= 128 ? 16 : gemm_ctas(bn, sums) == 2 ? 4 : 8; }
constexpr int gemm_threads(int epi) { return (epi + 4) * 32; }
static_assert(128 * 56 + 8 * 32 * 224 <= gemm_threads(8) * 168 && 128 * 32 + 16 * 32 * 112 <= gemm_threads(16) * 96,
              "registers of a CTA");
constexpr int kMaxRing = 16;
constexpr uint32_t kTileA = 128 * 128;  // 128 rows (or 2 x 64 columns) x 64 of the contraction
__host__ __device__ constexpr uint32_t gemm_main(int epi) { return (epi == 4 ? 108 : 224) * 1024; }    // bytes: rings and staging
__host__ __device__ constexpr uint32_t gemm_ring(int epi) { return gemm_main(epi) - epi * 4096; }  // 4 KB a warp to stage outputs
constexpr uint32_t kGemmBars = (6 * kMaxRing + 5) * 8 + 16;
constexpr uint32_t gemm_smem(int epi) { return 1024 + gemm_main(epi) + kGemmBars; }
static_assert(gemm_smem(8) <= 227 * 1024 && 2 * (gemm_smem(4) + 1024) <= 228 * 1024, "shared memory of the CTAs of an SM");
constexpr int kGroupM = 8;              // m tiles that share their B tiles in L2 (16: 1 % slower at 4096 x 1024 x 32003)
constexpr long long kDrain = 4000000000LL;  // clock cycles: waits for a CTA's own copies and MMAs before it ends

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void *tmap, int c0, int c1, int c2, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"((uint64_t)tmap), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
        : "memory");
}

// The same lane of a whole warp every time.
__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// mbar_wait by a whole warp, one answer for all of it.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, long long limit, volatile int *abort)
{
    if (__all_sync(0xffffffffu, tc::mbar_test_wait(bar, parity))) return true;
    const long long t0 = clock64();
    while (true) {
        if (__any_sync(0xffffffffu, clock64() - t0 >= limit || *abort)) return false;
        if (__all_sync(0xffffffffu, tc::mbar_try_wait(bar, parity))) return true;
    }
}

// ---- pairs of CTAs (cta_group::2): one MMA of 256 rows over both, issued by the pair's first CTA;
// each CTA holds its 128 rows of A, half of B's rows and its 128 rows of the accumulator.
template <int CG>
__device__ __forceinline__ void tmem_alloc_cg(uint32_t *dst, uint32_t ncols)
{
    if constexpr (CG == 1) {
        tc::tmem_alloc(dst, ncols);
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(ncols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void tmem_dealloc_cg(uint32_t addr, uint32_t ncols)
{
    if constexpr (CG == 1)
        tc::tmem_dealloc(addr, ncols);
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(ncols) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_cg(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t more)
{
    if constexpr (CG == 1)
        tc::mma_bf16(d, da, db, idesc, more);
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(da), "l"(db), "r"(idesc), "r"(more)
            : "memory");
}
// Arrive on the barrier (of both CTAs of a pair) when the MMAs so far are done.
template <int CG>
__device__ __forceinline__ void commit_cg(uint64_t *bar)
{
    if constexpr (CG == 1)
        tc::mma_commit(bar);
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
            "h"((uint16_t)3)
            : "memory");
}
// Arrive on the pair's first CTA's barrier. (What is handed over are operands and accumulators that
// only the asynchronous proxies read and write: no thread's reads are ordered after this, and
// acquire and release at cluster scope, which a wait would pay 700 to 900 cycles for each time,
// have nothing to order.)
__device__ __forceinline__ void arrive_first(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(tc::mapa(smem_u32(bar), 0)) : "memory");
}

__device__ __forceinline__ void prefetch_map(const void *tmap)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)tmap) : "memory");
}

// D [M][N] += sum over the pairs of A_i B_j^T. A CTA takes units (tile, split) blockIdx.x,
// + gridDim.x, ...; a unit's chunks go through accumulators of per_acc chunks each, two of them
// in turn in tensor memory: the output warps add one up in registers (and after the last finish the
// tile) while the MMAs fill the other. The tensor cores' fp32 additions cut, so an accumulator
// that fp32 results come from takes few of them (1.7e-8 of the result each: 1e-4 after 6012).
// A part is loaded once a chunk, whatever number of products it is in, small products first.
// MN-major operands: blocks of 64 columns, each 64 rows of 128 bytes.
// Bound by the tensor cores where the contraction is long: both products of the backward at 4096 x
// 1024 x 32003 bf16, with the 245 us of their parts, 1280 us, as pairs of CTAs on 256 x 256 tiles.
// Bound by its output warps where it is short: forward 65536 x 1024 x 1024, gelu, residual and pre, 146
// us, 15 rounds of tiles of 19 thousand cycles each, of which the MMAs take 8. Nothing is saturated there
// (16384 rows: tensor pipe 34 %, issue 42 %, shared memory's data banks 12 %): the warps wait, for
// loads most of all (2.8 of 11.9 cycles an instruction), then for instructions (1.6).
// bf16 results come from one accumulator, whatever K is: 1.7e-8 of it an MMA, 16 of K (2^-11.8 at K =
// 2^18, where a bf16 result is rounded by 2^-9).
template <int BN, bool A_MN, bool B_MN, int PA, int PB, int EPI, int CG>
__global__ void __launch_bounds__(gemm_threads(EPI), EPI == 4 ? 2 : 1)
gemm_parts(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
           const __grid_constant__ GemmArgs g)
{
    constexpr Pairs<PA, PB> P;
    constexpr int BR = BN / CG;  // rows of B that a CTA holds
    constexpr uint32_t kTileB = (uint32_t)BR * 128u;
    constexpr int COLS = BN / (EPI / 4), SEG = COLS < 32 ? COLS : 32;  // an output warp's columns
    constexpr uint32_t kRing = gemm_ring(EPI);
    constexpr bool JOINT = PA == 1 && PB == 1;      // A's and B's slots go together: one barrier for both
    constexpr bool SUMS = A_MN || B_MN || PB == 3;  // fp32 results: several accumulators to a tile
    constexpr uint32_t kCols = 2 * BN < 32 ? 32 : 2 * BN;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int SA = g.SA, SB = g.SB;
    const uint32_t ring_a = smem_u32(base), ring_b = ring_a + (uint32_t)SA * kTileA;
    uint64_t *full_a = (uint64_t *)(base + gemm_main(EPI));
    uint64_t *empty_a = full_a + kMaxRing, *full_b = empty_a + kMaxRing, *empty_b = full_b + kMaxRing;
    uint64_t *peer_a = empty_b + kMaxRing, *peer_b = peer_a + kMaxRing;  // the pair's other CTA's operands have landed
    uint64_t *acc_full = peer_b + kMaxRing, *acc_empty = acc_full + 2, *done = acc_empty + 2;
    uint32_t *tmem_slot = (uint32_t *)(done + 1);
    volatile int *abort = (volatile int *)(tmem_slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = CG == 1 ? 0 : (int)tc::cluster_rank();
    if (tid < kMaxRing) {  // (every ring's, used or not)
        tc::mbar_init(&full_a[tid], 1);
        tc::mbar_init(&empty_a[tid], 1);
        tc::mbar_init(&full_b[tid], 1);
        tc::mbar_init(&empty_b[tid], 1);
        tc::mbar_init(&peer_a[tid], 1);
        tc::mbar_init(&peer_b[tid], 1);
        if (tid < 2) {
            tc::mbar_init(&acc_full[tid], 1);
            tc::mbar_init(&acc_empty[tid], CG * EPI);
        }
        if (tid == 0) {
            tc::mbar_init(done, 1);
            *abort = 0;
        }
        tc::fence_mbar_init();
    }
    if (tid == 32) {
        prefetch_map(&tm_a);
        prefetch_map(&tm_b);
    }
    if (warp == 0) tmem_alloc_cg<CG>(tmem_slot, kCols);
    tc::tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) tc::cluster_sync();  // the other CTA's barriers are there
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    after_previous();
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
        m0 = (first + in % gm) * 128 * CG + rank * 128;  // (this CTA's rows)
        n0 = in / gm * (SUMS ? g.step : BN);
        c_lo = (int)((long long)g.chunks * sp / g.split);
        c_hi = (int)((long long)g.chunks * (sp + 1) / g.split);
    };
    // Columns that a tile's MMAs take. Tiles of fp32 results are as wide as one another, in steps of 16
    // (a pair of CTAs: 32), and their MMAs stop at the contraction's end: 11840 x 600 x 200 fp32
    // backward 77.5 us, 83.1 with tiles of 256, 256 and 88 and whole chunks. The rest of an accumulator is
    // not written, and no output is made of it. (bf16 forward: 65536 x 1024 x 1024 148 us so, 144 with
    // whole tiles; its MMAs are not what it waits for.)
    auto width = [&](int n0) {
        return SUMS ? (uint32_t)min(g.step, (g.N - n0 + 16 * CG - 1) / (16 * CG) * (16 * CG)) : (uint32_t)BN;
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

    if (warp < 4) {
        if constexpr (EPI == 8)
            asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        else if constexpr (EPI == 16)
            asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
        // Both loops are run by whole warps, one lane of which issues: descriptors and coordinates
        // are then the same for a warp and stay in its uniform registers (by one thread in a branch
        // of its own an MMA took 125 cycles to issue, whatever its size).
        const bool issues = elect_one();
        if (warp == 0) {
            long long na = 0, nb = 0;  // loads
            bool ok = true;
            for (long long u = blockIdx.x / CG; ok && u < units; u += gridDim.x / CG) {
                unit(u, m0, n0, sp, c_lo, c_hi);
                const int b0 = n0 + (CG == 2 ? rank * (int)width(n0) / 2 : 0);  // (this CTA's rows of B)
                for (int c = c_lo; ok && c < c_hi; ++c) {
                    const int k0 = c * 64;
#pragma unroll
                    for (int p = 0; p < P.n; ++p) {
                        if (P.load_b[p] && ok) {
                            const int at = P.at_b[P.b[p]], s = rb.slot(at);
                            ok = warp_wait(&empty_b[s], rb.phase(at) ^ 1, limit, abort);
                            if (ok) {
                                ++nb;
                                const uint32_t dst = ring_b + s * kTileB;
                                if (issues) {
                                    tc::mbar_arrive_expect_tx(&full_b[s], JOINT ? kTileA + kTileB : kTileB);
                                    if constexpr (B_MN) {
#pragma unroll
                                        for (int j = 0; j < BR / 64; ++j)
                                            tma_load_3d(dst + j * 8192, &tm_b, b0 + j * 64, k0, P.b[p], &full_b[s]);
                                    } else {
                                        tma_load_3d(dst, &tm_b, k0, b0, P.b[p], &full_b[s]);
                                    }
                                }
                            }
                        }
                        if (P.load_a[p] && ok) {
                            const int at = P.at_a[P.a[p]], s = ra.slot(at);
                            uint64_t *full = JOINT ? &full_b[s] : &full_a[s];
                            if (!JOINT) ok = warp_wait(&empty_a[s], ra.phase(at) ^ 1, limit, abort);
                            if (ok) {
                                if (!JOINT) ++na;
                                const uint32_t dst = ring_a + s * kTileA;
                                if (issues) {
                                    if (!JOINT) tc::mbar_arrive_expect_tx(full, kTileA);
                                    if constexpr (A_MN) {
                                        tma_load_3d(dst, &tm_a, m0, k0, P.a[p], full);
                                        tma_load_3d(dst + 8192, &tm_a, m0 + 64, k0, P.a[p], full);
                                    } else {
                                        tma_load_3d(dst, &tm_a, k0, m0, P.a[p], full);
                                    }
                                }
                            }
                        }
                    }
                    ra.next(PA);
                    rb.next(PB);
                }
            }
            if (!ok && issues) fail();
            // no copy in flight when the CTA ends: the last load of every slot has landed
            for (int s = 0; s < SA; ++s)
                if (na > s) tc::mbar_wait(&full_a[s], (uint32_t)((na - 1 - s) / SA) & 1, kDrain, nullptr);
            for (int s = 0; s < SB; ++s)
                if (nb > s) tc::mbar_wait(&full_b[s], (uint32_t)((nb - 1 - s) / SB) & 1, kDrain, nullptr);
        }
        if (warp == 1 && rank == 0) {
            const uint64_t desc_a = tc::smem_desc(ring_a, A_MN ? 8192 : 16, 1024), desc_b = tc::smem_desc(ring_b, B_MN ? 8192 : 16, 1024);
            uint32_t acc = 0;  // accumulators filled so far
            bool ok = true;
            for (long long u = blockIdx.x / CG; ok && u < units; u += gridDim.x / CG) {
                unit(u, m0, n0, sp, c_lo, c_hi);
                const uint32_t idesc = tc::idesc_bf16(width(n0), A_MN, B_MN, 128 * CG);
                for (int c = c_lo; ok && c < c_hi; ++acc) {
                    const uint32_t d = tmem + (acc & 1) * BN;
                    ok = warp_wait(&acc_empty[acc & 1], ((acc >> 1) & 1) ^ 1, limit, abort);
                    if (!ok) break;
                    tc::tc_fence_after();
                    const int c_end = min(c_hi, c + g.per_acc);
                    uint32_t more = 0;
                    for (; ok && c < c_end; ++c) {
                        const int left = g.K - c * 64;  // of the contraction: steps of 16 past its end are left out
#pragma unroll
                        for (int p = 0; p < P.n; ++p) {
                            const int ia = P.at_a[P.a[p]], ib = P.at_b[P.b[p]], sa = ra.slot(ia), sb = rb.slot(ib);
                            if (P.load_b[p] && ok) ok = warp_wait(&full_b[sb], rb.phase(ib), limit, abort);
                            if (P.load_a[p] && ok && !JOINT) ok = warp_wait(&full_a[sa], ra.phase(ia), limit, abort);
                            if (CG == 2 && P.load_b[p] && ok) ok = warp_wait(&peer_b[sb], rb.phase(ib), limit, abort);
                            if (CG == 2 && P.load_a[p] && ok && !JOINT) ok = warp_wait(&peer_a[sa], ra.phase(ia), limit, abort);
                            if (ok) {
                                const uint64_t da = desc_a + (uint32_t)sa * (kTileA >> 4), db = desc_b + (uint32_t)sb * (kTileB >> 4);
                                if (issues) {
#pragma unroll
                                    for (int k = 0; k < 4; ++k)  // 16 of the contraction: 32 bytes of a row, or 16 rows
                                        if (!SUMS || k == 0 || left > 16 * k)
                                            mma_cg<CG>(d, da + k * (A_MN ? 128 : 2), db + k * (B_MN ? 128 : 2), idesc, k || p ? 1 : more);
                                    if (P.free_a[p] && !JOINT) commit_cg<CG>(&empty_a[sa]);
                                    if (P.free_b[p]) commit_cg<CG>(&empty_b[sb]);
                                }
                                __syncwarp();
                            }
                        }
                        more = 1;
                        ra.next(PA);
                        rb.next(PB);
                    }
                    if (ok && issues) commit_cg<CG>(&acc_full[acc & 1]);
                    __syncwarp();
                }
            }
            if (!ok && issues) fail();
            if (issues) commit_cg<CG>(done);
            __syncwarp();
            tc::mbar_wait(done, 0, kDrain, nullptr);  // no MMA in flight when tensor memory is freed
        }
        if (CG == 2 && warp == 1 && rank == 1) {  // tells the pair's first CTA what has landed here
            bool ok = true;
            for (long long u = blockIdx.x / CG; ok && u < units; u += gridDim.x / CG) {
                unit(u, m0, n0, sp, c_lo, c_hi);
                for (int c = c_lo; ok && c < c_hi; ++c) {
#pragma unroll
                    for (int p = 0; p < P.n; ++p) {
                        const int ia = P.at_a[P.a[p]], ib = P.at_b[P.b[p]], sa = ra.slot(ia), sb = rb.slot(ib);
                        if (P.load_b[p] && ok) {
                            ok = warp_wait(&full_b[sb], rb.phase(ib), limit, abort);
                            if (ok && issues) arrive_first(&peer_b[sb]);
                        }
                        if (P.load_a[p] && ok && !JOINT) {
                            ok = warp_wait(&full_a[sa], ra.phase(ia), limit, abort);
                            if (ok && issues) arrive_first(&peer_a[sa]);
                        }
                    }
                    ra.next(PA);
                    rb.next(PB);
                }
            }
            if (!ok && issues) fail();
            tc::mbar_wait(done, 0, kDrain, nullptr);  // (the last arrivals here of the other CTA's MMAs)
        }
        __syncwarp();
    } else {
        if constexpr (EPI == 8)
            asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        else if constexpr (EPI == 16)
            asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
        // ------------------------------------------------------ sums and outputs
        const int q = warp & 3, group = (warp >> 2) - 1;  // a warp reads its quadrant of the lanes
        float *stage = (float *)(base + kRing) + (warp - 4) * 1024;
        uint32_t acc = 0;
        bool ok = true;
        for (long long u = blockIdx.x / CG; ok && u < units; u += gridDim.x / CG) {
            unit(u, m0, n0, sp, c_lo, c_hi);
            const int mm = m0 + q * 32, nn = n0 + group * COLS;
            float *mine = stage + lane * 32;
            // (the whole warp waits together: its reads of tensor memory are collective)
            auto filled = [&]() {
                const bool got = warp_wait(&acc_full[acc & 1], (acc >> 1) & 1, limit, abort);
                tc::tc_fence_after();
                return got;
            };
            auto release = [&]() {
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 1)
                        tc::mbar_arrive(&acc_empty[acc & 1]);
                    else
                        arrive_first(&acc_empty[acc & 1]);
                }
                ++acc;
            };
            auto read = [&](int col, uint32_t (&v)[SEG / 16][16]) {  // SEG columns, their reads in flight together
                const uint32_t at = tmem + ((uint32_t)(q * 32) << 16) + (acc & 1) * BN + group * COLS + col;
#pragma unroll
                for (int j = 0; j < SEG / 16; ++j) tc::tmem_ld16_async(at + 16 * j, v[j]);
                tc::tmem_wait_ld();
            };
            if constexpr (SUMS) {
                float sum[COLS];
#pragma unroll
                for (int i = 0; i < COLS; ++i) sum[i] = 0.0f;
#pragma unroll 1
                for (int c = c_lo; c < c_hi; c += g.per_acc) {
                    if (!(ok = filled())) break;
#pragma unroll
                    for (int i = 0; i < COLS; i += SEG) {
                        uint32_t v[SEG / 16][16];
                        read(i, v);
#pragma unroll
                        for (int j = 0; j < SEG; ++j) sum[i + j] += __uint_as_float(v[j / 16][j % 16]);
                    }
                    release();
                }
                if (!ok) break;
                auto in = [&](int seg) {
#pragma unroll
                    for (int k = 0; k < COLS / SEG; ++k)
                        if (seg == k)
#pragma unroll
                            for (int i = 0; i < SEG / 4; ++i) {
                                const float *v = sum + k * SEG + 4 * i;
                                *(float4 *)(mine + ((i ^ (lane & 7)) << 2)) = make_float4(v[0], v[1], v[2], v[3]);
                            }
                    return true;
                };
                put_tile<SEG, COLS / SEG, A_MN || B_MN, true>(in, g.ep, g.swapped, sp, stage, lane, mm, nn, min(g.N, n0 + g.step));
            } else {
                auto in = [&](int seg) {
                    if (seg == 0 && !filled()) return false;
                    uint32_t v[SEG / 16][16];
                    read(seg * SEG, v);
#pragma unroll
                    for (int i = 0; i < SEG / 4; ++i)
                        *(uint4 *)(mine + ((i ^ (lane & 7)) << 2)) =
                            make_uint4(v[i / 4][i % 4 * 4], v[i / 4][i % 4 * 4 + 1], v[i / 4][i % 4 * 4 + 2], v[i / 4][i % 4 * 4 + 3]);
                    if (seg == COLS / SEG - 1) release();
                    return true;
                };
                ok = put_tile<SEG, COLS / SEG, false, false>(in, g.ep, g.swapped, sp, stage, lane, mm, nn, 0);
            }
        }
        if (!ok && lane == 0) fail();
    }
    tc::tc_fence_before();
    __syncthreads();
    // (a pair's CTAs end together: one's MMAs read the other's operands, the other arrives on its barriers)
    if constexpr (CG == 2) tc::cluster_sync();
    if (warp == 0) tmem_dealloc_cg<CG>(tmem, kCols);
}

// The splits' sums of each output added in split order, then its epilogue.
template <typename Out>
__device__ __forceinline__ void join(const Epilogue &ep, int split, const Out &o)
{
    const size_t n = (size_t)ep.rows * ep.cols;
    for (size_t e = blockIdx.x * (size_t)256 + threadIdx.x; e < n; e += (size_t)gridDim.x * 256) {
        float v = 0.0f;
        if (n < (size_t)1 << 15) {  // few threads: the reads of sixteen in flight
            for (int s0 = 0; s0 < split; s0 += 16) {
                float w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = s0 + i < split ? ep.part[(size_t)(s0 + i) * n + e] : 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) v += w[i];
            }
        } else {
#pragma unroll 4
            for (int s = 0; s < split; ++s) v += ep.part[(size_t)s * n + e];
        }
        o.put(e, v, ep.bias ? ep.bias[e % ep.cols] : 0.0f, o.extra(e));
    }
}
__global__ void __launch_bounds__(256)
join_splits(const __grid_constant__ Epilogue ep, int split)
{
    after_previous();
    if (ep.out)
        join(ep, split, Plain{ep.add, ep.out});
    else if (ep.bf16_out)
        join(ep, split, Forward<__nv_bfloat16>(ep));
    else
        join(ep, split, Forward<float>(ep));
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

template <int BN, bool A_MN, bool B_MN, int PA, int PB, int CG>
cudaError_t launch_gemm(const stacklstm_op *op, const Operand &a, const Operand &b, const GemmArgs &g)
{
    CUtensorMap ta, tb;
    cudaError_t e = operand_map(&ta, a, A_MN ? 64 : 128);
    if (!e) e = operand_map(&tb, b, B_MN ? 64 : BN / CG);
    constexpr int EPI = gemm_epi_warps(BN, A_MN || B_MN || PB == 3);
    constexpr auto kernel = gemm_parts<BN, A_MN, B_MN, PA, PB, EPI, CG>;
    if (!e) e = smem_at_least((const void *)kernel, gemm_smem(EPI));
    if (e) return e;
    const int most = CG == 2 ? op->pairs : op->num_sms * gemm_ctas(BN, A_MN || B_MN || PB == 3);
    const unsigned grid = (unsigned)std::min<long long>((long long)g.mt * g.nt * g.split, most) * CG;
    return launch_cluster(kernel, CG, grid, gemm_threads(EPI), gemm_smem(EPI), op->stream, ta, tb, g);
}

// Pairs of CTAs that run at once: fewer than half the SMs where a group of SMs has an odd number of
// them in use (76 pairs in a grid of which 72 run at once took twice the time).
int most_pairs()
{
    constexpr auto kernel = gemm_parts<256, false, false, 1, 1, gemm_epi_warps(256, false), 2>;
    if (smem_at_least((const void *)kernel, gemm_smem(16))) return 0;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 2;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2);
    cfg.blockDim = dim3(gemm_threads(gemm_epi_warps(256, false)));
    cfg.dynamicSmemBytes = gemm_smem(16);
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int n = 0;
    return cudaOccupancyMaxActiveClusters(&n, (const void *)kernel, &cfg) == cudaSuccess ? n : 0;
}

enum { kWsX = 0, kWsW, kWsDz, kWsSum, kWsPart, kWsCount };  // workspace buffers

constexpr size_t kMostPartBytes = (size_t)1 << 30;  // of the splits' sums

// One CTA a tile of 128 rows or a pair a tile of 256, the tile's width, and the splits: the least of
// waves x chunks x cycles a chunk, a tile's start and end, and for a split contraction its sums
// written and read again, and a second launch. A chunk takes two cycles a column and product, or
// what shared memory takes for the operands (128 bytes a cycle: written once a part, read once a
// product), which is more for one CTA: 16 + 32 KB read a product of 128 x 256, 16 + 16 by each of
// a pair.
struct GemmPlan {
    int cg, bn;
};
GemmPlan plan_gemm(GemmArgs &g, int PA, int PB, int npair, int M, int N, int bn_lo, int bn_hi, size_t out_elems, int sms, int pairs)
{
    GemmPlan best_plan = {1, 64};
    double best = 1e300;
    for (int cg = 1; cg <= (pairs ? 2 : 1); ++cg)
        for (int bn = bn_lo; bn <= bn_hi; bn *= 2) {
            if (cg == 2 ? bn != 256 : bn == 256 && PB == 3) continue;  // (no such kernels)
            const int step = PA > 1 ? 16 * cg * ceil_div(N, (size_t)16 * cg * ceil_div(N, bn)) : bn;
            const double mt = ceil_div(M, 128 * cg), nt = ceil_div(N, step), b = bn * 128.0 / cg;
            const double smem = (npair * (kTileA + step * 128.0 / cg) + PA * (double)kTileA + PB * b) / 128.0;
            const int ctas = cg == 2 ? pairs : sms * gemm_ctas(bn, PA > 1);
            const double cyc = std::max(2.0 * step * npair, smem) * (cg == 2 ? 1 : ctas / sms);
            for (int split = 1; split <= std::min(g.chunks, 64); ++split) {
                if (split > 1 && (g.chunks / split < 2 || (double)split * out_elems * 4 > (double)kMostPartBytes)) break;
                const double waves = std::ceil(mt * nt * split / ctas), chunks = std::ceil((double)g.chunks / split);
                double cost = waves * ((split > 1 || PA == 1 ? chunks : ceil_div(g.K, 16) / 4.0) * cyc + 400.0) + 16.0 * bn + 2000.0 + 1000.0 * cg;
                if (split > 1) cost += 5000.0 + 2.0 * split * out_elems * 4 / 3500.0;
                if (cost < best) {
                    best = cost;
                    g.mt = (int)mt;
                    g.nt = (int)nt;
                    g.step = step;
                    g.split = split;
                    best_plan = {cg, bn};
                }
            }
        }
    return best_plan;
}

// D = sum over the parts' products of A B^T, kcols long, and its epilogue.
template <bool A_MN, bool B_MN, int PA, int PB>
cudaError_t contract_parts(stacklstm_op *op, const Operand &a, const Operand &b, int kcols, bool swapped, Epilogue ep)
{
    constexpr Pairs<PA, PB> P;
    GemmArgs g = {};
    g.K = kcols;
    g.chunks = (int)ceil_div(kcols, 64);
    // fp32 results: 24 or 36 MMAs to an accumulator (24 everywhere: 4096 x 1024 x 32003 backward 1294 us, 1263 so)
    g.per_acc = ep.out || !ep.bf16_out ? std::max(1, 9 / P.n) : g.chunks;
    g.swapped = swapped;
    g.limit = op->wait_limit;
    g.err = op->err;
    const int M = swapped ? ep.cols : ep.rows, N = swapped ? ep.rows : ep.cols;
    const int lo = swapped && N <= 32 ? 32 : 64, hi = N <= lo ? lo : N <= 64 ? 64 : N <= 128 ? 128 : 256;
    g.N = N;
    const GemmPlan plan = plan_gemm(g, PA, PB, P.n, M, N, lo, hi, (size_t)ep.rows * ep.cols, op->num_sms, op->pairs);
    const int bn = plan.bn;
    // rings: as many whole chunks as fit, what is left to the single part of B, then to A
    const uint32_t tb = (uint32_t)bn * 128 / plan.cg;
    const uint32_t ring = gemm_ring(gemm_epi_warps(bn, A_MN || B_MN || PB == 3));
    const int depth = (int)(ring / (PA * kTileA + PB * tb));
    g.SA = std::min(kMaxRing / PA, depth) * PA;
    g.SB = std::min(kMaxRing / PB, depth) * PB;
    while (g.SB < kMaxRing && g.SA * kTileA + (g.SB + 1) * tb <= ring && PB < PA) ++g.SB;
    while (PA > 1 && g.SA < kMaxRing && (g.SA + 1) * kTileA + g.SB * tb <= ring) ++g.SA;
    if (g.split > 1) {
        cudaError_t e = op_workspace(op, kWsPart, (size_t)g.split * ep.rows * ep.cols * 4);
        if (e) return e;
        ep.part = (float *)op->ws[kWsPart];
    }
    g.ep = ep;
    cudaError_t e = cudaErrorInvalidValue;
    if constexpr (!A_MN && !B_MN)
        if (bn == 32) e = launch_gemm<32, A_MN, B_MN, PA, PB, 1>(op, a, b, g);
    if (bn == 64) e = launch_gemm<64, A_MN, B_MN, PA, PB, 1>(op, a, b, g);
    if (bn == 128) e = launch_gemm<128, A_MN, B_MN, PA, PB, 1>(op, a, b, g);
    if (bn == 256 && plan.cg == 2) e = launch_gemm<256, A_MN, B_MN, PA, PB, 2>(op, a, b, g);
    if constexpr (PB == 1)  // (three parts of a 256-wide B leave one CTA's rings no second chunk)
        if (bn == 256 && plan.cg == 1) e = launch_gemm<256, A_MN, B_MN, PA, PB, 1>(op, a, b, g);
    if (!e && g.split > 1) {
        const unsigned ctas = (unsigned)std::min<size_t>(ceil_div((size_t)ep.rows * ep.cols, 256), (size_t)op->num_sms * 8);
        e = launch_after(join_splits, ctas, 256, 0, op->stream, ep, g.split);
    }
    return e;
}

// (x and W have the parts of their type, dz always three)
template <bool A_MN, bool B_MN>
cudaError_t contract(stacklstm_op *op, const Operand &a, const Operand &b, int kcols, bool swapped, const Epilogue &ep)
{
    if (b.parts == 3) return contract_parts<A_MN, B_MN, 3, 3>(op, a, b, kcols, swapped, ep);
    if constexpr (A_MN || B_MN)
        return contract_parts<A_MN, B_MN, 3, 1>(op, a, b, kcols, swapped, ep);
    else
        return contract_parts<A_MN, B_MN, 1, 1>(op, a, b, kcols, swapped, ep);
}

int row_ld(int cols) { return (cols + 7) / 8 * 8; }

// An activation or weight tensor as an operand: itself where its rows start on 16 bytes, else what
// `pack` makes of it in the workspace (a copy, or the three parts of an fp32 one).
cudaError_t as_operand(stacklstm_op *op, const void *src, size_t rows, int cols, int ws, Pack *pack, Operand *o)
{
    const int ld = row_ld(cols);
    if (op->dt == SL_BF16 && ld == cols) {
        *o = {src, rows, cols, cols, 1};
        return cudaSuccess;
    }
    const int parts = op->dt == SL_BF16 ? 1 : 3;
    if (cudaError_t e = op_workspace(op, ws, (size_t)parts * rows * ld * 2)) return e;
    *pack = {src, (__nv_bfloat16 *)op->ws[ws], rows, cols, ld, ceil_div(rows * ld / 4, 256 * kPackItems)};
    *o = {op->ws[ws], rows, cols, ld, parts};
    return cudaSuccess;
}

cudaError_t launch_prepare(const stacklstm_op *op, const Prepare &p)
{
    const unsigned ctas = p.dz.ctas + p.x.ctas + p.w.ctas;
    if (!ctas) return cudaSuccess;
    return op->dt == SL_BF16 ? launch_after(prepare<__nv_bfloat16>, ctas, 256, 0, op->stream, p)
                             : launch_after(prepare<float>, ctas, 256, 0, op->stream, p);
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
    OpDevice guard(device);
    const size_t counts = ceil_div(N, kDzCols) * 4;
    op->pairs = most_pairs();
    if (op_workspace(op, kWsCount, counts) || cudaMemsetAsync(op->ws[kWsCount], 0, counts, op->stream)) {
        cudaGetLastError();
        stacklstm_op_destroy(op);
        return SL_ERR_OOM;
    }
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
    Prepare p = {};
    cudaError_t e = as_operand(op, x, rows, op->K, kWsX, &p.x, &xo);
    if (!e) e = as_operand(op, W, op->N, op->K, kWsW, &p.w, &wo);
    if (!e) e = launch_prepare(op, p);
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
    // dz in parts, its column sums; the operands
    Prepare p = {};
    Operand dz = {nullptr, (size_t)rows, N, row_ld(N), 3}, wo, xo;
    if (dx || dW) e = op_workspace(op, kWsDz, 3 * (size_t)rows * dz.ld * 2);
    p.dz.row_blocks = ceil_div(rows, kDzRows);
    if (!e && dbias) e = op_workspace(op, kWsSum, (size_t)p.dz.row_blocks * N * 4);
    if (!e && dx) e = as_operand(op, W, N, K, kWsW, &p.w, &wo);
    if (!e && dW) e = as_operand(op, x, rows, K, kWsX, &p.x, &xo);
    if (!e && (dx || dW || dbias)) {
        if (dx || dW) dz.p = op->ws[kWsDz];
        p.dz.dy = dy; p.dz.pre = pre; p.dz.out = (__nv_bfloat16 *)dz.p; p.dz.part = dbias ? (float *)op->ws[kWsSum] : nullptr;
        p.dz.dbias = dbias; p.dz.arrived = (int *)op->ws[kWsCount]; p.dz.rows = rows; p.dz.N = N; p.dz.ld = dz.ld; p.dz.act = op->act;
        p.dz.ctas = p.dz.row_blocks * ceil_div(N, kDzCols);
        for (p.dz.lanes = 32; p.dz.lanes > 1 && 2 * N <= 4 * p.dz.lanes; p.dz.lanes /= 2) {}
        e = launch_prepare(op, p);
    }
    if (!e && dx) {
        Epilogue ep = {};
        ep.rows = rows; ep.cols = K; ep.out = dx; ep.add = add;
        e = contract<false, true>(op, dz, wo, N, false, ep);
    }
    if (!e && dW) {
        Epilogue ep = {};
        ep.rows = N; ep.cols = K; ep.out = dW;
        e = contract<true, true>(op, dz, xo, rows, false, ep);
    }
    return e ? op_cuda(op, e, "stacklstm_linear_backward") : SL_OK;
}

}  // extern "C"
