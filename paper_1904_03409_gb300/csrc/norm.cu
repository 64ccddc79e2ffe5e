// norm.cu -- layer norm of the StackLSTM outputs, forward and backward, and its C ABI
// (include/stacklstm.h, stacklstm_norm_*).
//
// Row r of x [rows][N]: m = mean(x), s = (mean((x - m)^2) + eps)^(-1/2), xh = (x - m) s,
// y = xh gamma + beta. With a = dy gamma the backward is
//   dx = s (a - mean(a) - xh mean(a xh)),  dgamma = sum_r dy xh,  dbeta = sum_r dy.
// Both are bound by HBM: each tensor is read or written once. A row's elements stay in the
// registers of its threads (a warp, or a CTA of 256), so the variance is taken of the centred
// values and nothing is read twice; only rows wider than the registers hold (norm_*_wide) are
// read again, from the caches. The backward's CTAs keep their columns' sums of dgamma and dbeta
// in registers over all their rows and write them once; a second launch adds the CTAs' sums in
// CTA order, so the gradients are bitwise reproducible. (Products that a sum follows are rounded
// by __fmul_rn where a null output would otherwise let the compiler fuse the two, and change bits.)
#include "op.cuh"

namespace sl {
namespace {

constexpr int kNormThreads = 256;

// The TPR threads of a row hold CH pieces of VEC elements each: piece j of thread t is at column
// (j TPR + t) VEC.
template <typename T, int VEC, int CH, int TPR>
__global__ void __launch_bounds__(kNormThreads)
norm_fwd(int rows, int N, const T *__restrict__ x, const float *__restrict__ gamma, const float *__restrict__ beta,
         float eps, T *__restrict__ y, float *__restrict__ mean, float *__restrict__ rstd)
{
    constexpr int RPB = kNormThreads / TPR;
    __shared__ float sm[kNormThreads / 32];
    const int t = threadIdx.x % TPR;
    const float inv = 1.0f / (float)N;
    for (int r = blockIdx.x * RPB + threadIdx.x / TPR; r < rows; r += gridDim.x * RPB) {
        const size_t at = (size_t)r * N;
        float v[CH][VEC];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + t) * VEC;
            if (c < N) {
                load_vec<T, VEC>(x + at + c, v[j]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum += v[j][i];
            }
        }
        const float m = __fmul_rn(row_sum<TPR>(sum, sm), inv);
        float sq = 0.0f;
#pragma unroll
        for (int j = 0; j < CH; ++j)
            if ((j * TPR + t) * VEC < N)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[j][i] -= m;
                    sq = fmaf(v[j][i], v[j][i], sq);
                }
        const float s = 1.0f / sqrtf(row_sum<TPR>(sq, sm) * inv + eps);
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + t) * VEC;
            if (c < N) {
                float g[VEC], b[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    g[i] = 1.0f;
                    b[i] = 0.0f;
                }
                if (gamma) load_vec<float, VEC>(gamma + c, g);
                if (beta) load_vec<float, VEC>(beta + c, b);
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[j][i] = fmaf(v[j][i] * s, g[i], b[i]);
                store_vec<T, VEC>(y + at + c, v[j]);
            }
        }
        if (t == 0) {
            if (mean) mean[r] = m;
            if (rstd) rstd[r] = s;
        }
    }
}

// Rows of any width: a CTA a row, three passes over it (the last two from the caches).
template <typename T>
__global__ void __launch_bounds__(kNormThreads)
norm_fwd_wide(int rows, int N, const T *__restrict__ x, const float *__restrict__ gamma,
              const float *__restrict__ beta, float eps, T *__restrict__ y, float *__restrict__ mean,
              float *__restrict__ rstd)
{
    __shared__ float sm[kNormThreads / 32];
    const float inv = 1.0f / (float)N;
    for (int r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *xr = x + (size_t)r * N;
        float sum = 0.0f, sq = 0.0f;
        for (int c = threadIdx.x; c < N; c += kNormThreads) sum += to_f32(xr[c]);
        const float m = __fmul_rn(row_sum<kNormThreads>(sum, sm), inv);
        for (int c = threadIdx.x; c < N; c += kNormThreads) {
            const float d = to_f32(xr[c]) - m;
            sq = fmaf(d, d, sq);
        }
        const float s = 1.0f / sqrtf(row_sum<kNormThreads>(sq, sm) * inv + eps);
        for (int c = threadIdx.x; c < N; c += kNormThreads)
            y[(size_t)r * N + c] = from_f32<T>(fmaf((to_f32(xr[c]) - m) * s, gamma ? gamma[c] : 1.0f, beta ? beta[c] : 0.0f));
        if (threadIdx.x == 0) {
            if (mean) mean[r] = m;
            if (rstd) rstd[r] = s;
        }
    }
}

// part [gridDim.x][2][N]: this CTA's sums of dy xh and dy over its rows.
template <typename T, int VEC, int CH, int TPR>
__global__ void __launch_bounds__(kNormThreads)
norm_bwd(int rows, int N, const float *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ gamma,
         const float *__restrict__ mean, const float *__restrict__ rstd, float *__restrict__ dx,
         float *__restrict__ part)
{
    constexpr int RPB = kNormThreads / TPR;
    __shared__ float sm[kNormThreads / 32];
    extern __shared__ float cols[];  // [RPB][N] when RPB > 1: the warps' column sums
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const float inv = 1.0f / (float)N;
    float dg[CH][VEC], db[CH][VEC];
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) dg[j][i] = db[j][i] = 0.0f;
    for (int r = blockIdx.x * RPB + sub; r < rows; r += gridDim.x * RPB) {
        const size_t at = (size_t)r * N;
        const float m = mean[r], s = rstd[r];
        float a[CH][VEC], xh[CH][VEC];
        float sa = 0.0f, sx = 0.0f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + t) * VEC;
            if (c < N) {
                float g[VEC];
                load_vec<float, VEC>(dy + at + c, a[j]);
                load_vec<T, VEC>(x + at + c, xh[j]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] = 1.0f;
                if (gamma) load_vec<float, VEC>(gamma + c, g);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    xh[j][i] = __fmul_rn(xh[j][i] - m, s);
                    dg[j][i] = fmaf(a[j][i], xh[j][i], dg[j][i]);
                    db[j][i] += a[j][i];
                    a[j][i] = __fmul_rn(a[j][i], g[i]);
                    sa += a[j][i];
                    sx = fmaf(a[j][i], xh[j][i], sx);
                }
            }
        }
        if (dx) {
            const float ma = __fmul_rn(row_sum<TPR>(sa, sm), inv), mx = __fmul_rn(row_sum<TPR>(sx, sm), inv);
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int c = (j * TPR + t) * VEC;
                if (c < N) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) a[j][i] = s * (a[j][i] - ma - xh[j][i] * mx);
                    store_vec<float, VEC>(dx + at + c, a[j]);
                }
            }
        }
    }
    if (!part) return;
    float *out = part + (size_t)blockIdx.x * 2 * N;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (RPB > 1) __syncthreads();
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + t) * VEC;
            if (c < N)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float v = which ? db[j][i] : dg[j][i];
                    if constexpr (RPB > 1)
                        cols[(size_t)sub * N + c + i] = v;
                    else
                        out[(size_t)which * N + c + i] = v;
                }
        }
        if constexpr (RPB > 1) {
            __syncthreads();
            for (int c = threadIdx.x; c < N; c += kNormThreads) {
                float acc = 0.0f;
#pragma unroll
                for (int w = 0; w < RPB; ++w) acc += cols[(size_t)w * N + c];
                out[(size_t)which * N + c] = acc;
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kNormThreads)
norm_bwd_wide(int rows, int N, const float *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ gamma,
              const float *__restrict__ mean, const float *__restrict__ rstd, float *__restrict__ dx,
              float *__restrict__ part)
{
    __shared__ float sm[kNormThreads / 32];
    const float inv = 1.0f / (float)N;
    float *out = part ? part + (size_t)blockIdx.x * 2 * N : nullptr;
    if (out)
        for (int c = threadIdx.x; c < 2 * N; c += kNormThreads) out[c] = 0.0f;
    __syncthreads();
    for (int r = blockIdx.x; r < rows; r += gridDim.x) {
        const float *dr = dy + (size_t)r * N;
        const T *xr = x + (size_t)r * N;
        const float m = mean[r], s = rstd[r];
        float sa = 0.0f, sx = 0.0f;
        for (int c = threadIdx.x; c < N; c += kNormThreads) {
            const float a = dr[c] * (gamma ? gamma[c] : 1.0f);
            sa += a;
            sx = fmaf(a, (to_f32(xr[c]) - m) * s, sx);
        }
        const float ma = row_sum<kNormThreads>(sa, sm) * inv, mx = row_sum<kNormThreads>(sx, sm) * inv;
        for (int c = threadIdx.x; c < N; c += kNormThreads) {
            const float d = dr[c], xh = (to_f32(xr[c]) - m) * s;
            if (dx) dx[(size_t)r * N + c] = s * (d * (gamma ? gamma[c] : 1.0f) - ma - xh * mx);
            if (out) {  // a thread owns its columns: no other thread of the CTA touches them
                const int o = c;
                out[o] = fmaf(d, xh, out[o]);
                out[N + o] += d;
            }
        }
    }
}

// dgamma, dbeta = the parts' sums in part order: warp w of a CTA adds parts w, w + 8, ... of 32
// columns, then the eight sums are added in order.
__global__ void __launch_bounds__(256)
norm_reduce(const float *__restrict__ part, int n, int N, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    __shared__ float sm[8][32];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const size_t c = blockIdx.x * (size_t)32 + lane, W = 2 * (size_t)N;
    float acc = 0.0f;
    if (c < W) {
#pragma unroll 8
        for (int s = w; s < n; s += 8) acc += part[(size_t)s * W + c];
    }
    sm[w][lane] = acc;
    __syncthreads();
    if (w == 0 && c < W) {
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += sm[i][lane];
        if (c < (size_t)N) {
            if (dgamma) dgamma[c] = v;
        } else if (dbeta) {
            dbeta[c - N] = v;
        }
    }
}

// Pieces a thread holds for a row of N elements over TPR threads (0: more than 4).
int pieces(int N, int vec, int tpr)
{
    const int n = (int)ceil_div((size_t)N, (size_t)vec * tpr);
    return n <= 1 ? 1 : n <= 2 ? 2 : n <= 4 ? 4 : 0;
}

template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

struct NormCall {
    stacklstm_op *op;
    int rows;
    const void *x;
    const float *gamma, *beta;
    float eps;
    void *y;
    float *mean, *rstd;
    // backward
    const float *dy;
    float *dx, *part;
    int grid;
};

template <typename T, int VEC, int CH, int TPR>
cudaError_t launch_norm(const NormCall &c)
{
    constexpr int RPB = kNormThreads / TPR;
    const int N = c.op->N;
    if (!c.dy) {
        norm_fwd<T, VEC, CH, TPR><<<c.grid, kNormThreads, 0, c.op->stream>>>(c.rows, N, (const T *)c.x, c.gamma, c.beta,
                                                                             c.eps, (T *)c.y, c.mean, c.rstd);
    } else {
        const size_t smem = RPB > 1 ? (size_t)RPB * N * 4 : 0;
        norm_bwd<T, VEC, CH, TPR><<<c.grid, kNormThreads, smem, c.op->stream>>>(
            c.rows, N, c.dy, (const T *)c.x, c.gamma, c.mean, c.rstd, c.dx, c.part);
    }
    return cudaGetLastError();
}

template <typename T>
cudaError_t dispatch_norm(const NormCall &c, int vec, int ch, int tpr)
{
    constexpr int V = kVec<T>;
#define SL_NORM(v, n, t) \
    if (vec == v && ch == n && tpr == t) return launch_norm<T, v, n, t>(c);
    SL_NORM(V, 1, 32) SL_NORM(V, 2, 32) SL_NORM(V, 4, 32) SL_NORM(V, 1, 256) SL_NORM(V, 2, 256) SL_NORM(V, 4, 256)
    SL_NORM(1, 1, 32) SL_NORM(1, 2, 32) SL_NORM(1, 4, 32) SL_NORM(1, 1, 256) SL_NORM(1, 2, 256) SL_NORM(1, 4, 256)
#undef SL_NORM
    if (!c.dy)
        norm_fwd_wide<T><<<c.grid, kNormThreads, 0, c.op->stream>>>(c.rows, c.op->N, (const T *)c.x, c.gamma, c.beta, c.eps,
                                                                    (T *)c.y, c.mean, c.rstd);
    else
        norm_bwd_wide<T><<<c.grid, kNormThreads, 0, c.op->stream>>>(c.rows, c.op->N, c.dy, (const T *)c.x, c.gamma,
                                                                    c.mean, c.rstd, c.dx, c.part);
    return cudaGetLastError();
}

// Pieces of 16 bytes where every row starts on 16 bytes of all its tensors, else single
// elements; a warp a row where four pieces a lane hold it, else a CTA.
cudaError_t run_norm(NormCall c)
{
    const stacklstm_op *op = c.op;
    const int vmax = op->dt == SL_BF16 ? 8 : 4;
    const int vec = op->N % vmax == 0 ? vmax : 1;
    int tpr = 32, ch = pieces(op->N, vec, 32);
    if (!ch) {
        tpr = 256;
        ch = pieces(op->N, vec, 256);
    }
    const int rpb = kNormThreads / tpr;
    c.grid = (int)std::min<size_t>(ceil_div((size_t)c.rows, (size_t)rpb), (size_t)op->num_sms * 4);
    return op->dt == SL_BF16 ? dispatch_norm<__nv_bfloat16>(c, vec, ch, tpr) : dispatch_norm<float>(c, vec, ch, tpr);
}

}  // namespace
}  // namespace sl

using namespace sl;

extern "C" {

sl_status stacklstm_norm_create(stacklstm_op_t *out, int R, int N, sl_dtype dtype, int device, void *stream)
{
    if (!out) return SL_ERR_ARG;
    *out = nullptr;
    if (R < 1 || N < 1 || (dtype != SL_FP32 && dtype != SL_BF16)) return SL_ERR_ARG;
    if (N > (1 << 24)) return SL_ERR_UNSUPPORTED;
    sl_status st;
    stacklstm_op *op = op_new(SL_OP_NORM, dtype, device, stream, &st);
    if (!op) return st;
    op->R = R;
    op->N = N;
    OpDevice guard(device);
    // the column sums of every CTA of a backward
    const size_t ctas = std::min<size_t>((size_t)R, (size_t)op->num_sms * 4);
    if (op_workspace(op, 0, ctas * 2 * (size_t)N * 4) != cudaSuccess) {
        stacklstm_op_destroy(op);
        return SL_ERR_OOM;
    }
    *out = op;
    return SL_OK;
}

sl_status stacklstm_norm_forward(stacklstm_op_t op, int rows, const void *x, const float *gamma, const float *beta,
                                 float eps, void *y, float *mean, float *rstd)
{
    if (!op || op->kind != SL_OP_NORM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (rows < 0 || rows > op->R) return op_fail(op, SL_ERR_ARG, "rows outside 0 .. R");
    if (!(eps >= 0.0f)) return op_fail(op, SL_ERR_ARG, "eps must not be negative");
    if (rows == 0) return SL_OK;
    if (const char *m = check_pointers({x, y}, {gamma, beta, mean, rstd})) return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    NormCall c = {};
    c.op = op; c.rows = rows; c.x = x; c.gamma = gamma; c.beta = beta; c.eps = eps; c.y = y; c.mean = mean; c.rstd = rstd;
    const cudaError_t e = run_norm(c);
    return e ? op_cuda(op, e, "stacklstm_norm_forward") : SL_OK;
}

sl_status stacklstm_norm_backward(stacklstm_op_t op, int rows, const float *dy, const void *x, const float *gamma,
                                  const float *mean, const float *rstd, float *dx, float *dgamma, float *dbeta)
{
    if (!op || op->kind != SL_OP_NORM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (rows < 0 || rows > op->R) return op_fail(op, SL_ERR_ARG, "rows outside 0 .. R");
    if (const char *m = check_pointers({}, {dx, dgamma, dbeta})) return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    cudaError_t e = cudaSuccess;
    if (rows == 0) {  // sums of nothing
        for (float *p : {dgamma, dbeta})
            if (p && !e) e = cudaMemsetAsync(p, 0, (size_t)op->N * 4, op->stream);
        return e ? op_cuda(op, e, "stacklstm_norm_backward") : SL_OK;
    }
    if (const char *m = check_pointers({dy, x, mean, rstd}, {gamma})) return op_fail(op, SL_ERR_ARG, m);
    NormCall c = {};
    c.op = op; c.rows = rows; c.x = x; c.gamma = gamma; c.mean = const_cast<float *>(mean);
    c.rstd = const_cast<float *>(rstd); c.dy = dy; c.dx = dx;
    const bool sums = dgamma || dbeta;
    c.part = sums ? (float *)op->ws[0] : nullptr;
    e = run_norm(c);
    if (!e && sums) {
        const int vmax = op->dt == SL_BF16 ? 8 : 4, vec = op->N % vmax == 0 ? vmax : 1;
        const int rpb = pieces(op->N, vec, 32) ? kNormThreads / 32 : 1;
        const int n = (int)std::min<size_t>(ceil_div((size_t)rows, (size_t)rpb), (size_t)op->num_sms * 4);
        norm_reduce<<<ceil_div(2 * (size_t)op->N, 32), 256, 0, op->stream>>>((const float *)op->ws[0], n, op->N, dgamma, dbeta);
        e = cudaGetLastError();
    }
    return e ? op_cuda(op, e, "stacklstm_norm_backward") : SL_OK;
}

}  // extern "C"
