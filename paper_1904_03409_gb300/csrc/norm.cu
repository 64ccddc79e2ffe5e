// norm.cu -- layer norm of the StackLSTM outputs, forward and backward, and its C ABI
// (include/stacklstm.h, stacklstm_norm_*).
//
// Row r of x [rows][N]: m = mean(x), s = (mean((x - m)^2) + eps)^(-1/2), xh = (x - m) s,
// y = xh gamma + beta. With a = dy gamma the backward is
//   dx = s (a - mean(a) - xh mean(a xh)),  dgamma = sum_r dy xh,  dbeta = sum_r dy.
// Both are bound by HBM: each tensor is read or written once. A row's elements stay in the
// registers of its threads (a warp, or a CTA of 256), so the variance is taken of the centred
// values and nothing is read twice, and the next row's are read while one is worked on; only rows
// wider than the registers hold (norm_*_wide) are read again, from the caches. The forward of 65536 x
// 1024 bf16, in a loop of its own, takes 50 us (5.4 TB/s), the backward 111 (6.0). The backward's CTAs keep their columns' sums of dgamma and dbeta
// in registers over all their rows and write them once; a second launch adds the CTAs' sums in
// CTA order, so the gradients are bitwise reproducible. (Products that a sum follows are rounded
// by __fmul_rn where a null output would otherwise let the compiler fuse the two, and change bits.)
#include "rowvec.cuh"
#include "tc.cuh"

namespace sl {
namespace {

// A row's TPR threads (a warp: CTAs of four rows, or a CTA of 256) hold CH pieces of VEC elements
// each: piece j of thread t is at column (j TPR + t) VEC. VEC = 16 bytes of the type where every
// row starts on 16 bytes, else 1, whose accesses of 2 or 4 bytes bound such rows: 65536 x 1023 bf16
// takes 122 and 297 us (forward, backward), 16384 x 4099 on the wide kernels 100 and 424.
constexpr int kWideThreads = 256;
__host__ __device__ constexpr int norm_threads(int tpr) { return tpr == 32 ? 128 : 256; }
// CTAs an SM of the forward: as many as their registers allow (the next row's pieces stay in them)
__host__ __device__ constexpr int norm_ctas(int tpr, int elems)
{
    return tpr == 32 ? (elems <= 16 ? 8 : 6) : (elems <= 16 ? 4 : 3);
}

// VEC fp32 values (whole: their address is on 32 bytes).
template <int VEC>
__device__ __forceinline__ void load_f32(const float *p, bool whole, float *v)
{
    if constexpr (VEC == 8)
        load8(p, whole, v);
    else
        load_vec<float, VEC>(p, v);
}
template <int VEC>
__device__ __forceinline__ void store_f32(float *p, bool whole, const float *v)
{
    if constexpr (VEC == 8)
        store8(p, whole, v);
    else
        store_vec<float, VEC>(p, v);
}

// A piece as it lies in memory.
template <typename T, int VEC>
struct Piece {
    uint4 q[VEC * sizeof(T) / 16];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < (int)(VEC * sizeof(T) / 16); ++i) q[i] = ((const uint4 *)p)[i];
    }
    __device__ __forceinline__ void get(float (&v)[VEC]) const
    {
        constexpr int E = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < VEC / E; ++i) {
            float w[E];
            unpack<T>(q[i], w);
#pragma unroll
            for (int k = 0; k < E; ++k) v[i * E + k] = w[k];
        }
    }
};
template <typename T>
struct Piece<T, 1> {
    T e;
    __device__ __forceinline__ void load(const T *p) { e = *p; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_f32(e); }
};

template <typename T, int VEC, int CH, int TPR>
__global__ void __launch_bounds__(norm_threads(TPR), norm_ctas(TPR, CH * VEC))
norm_fwd(unsigned rows, int N, const T *__restrict__ x, const float *__restrict__ gamma, const float *__restrict__ beta,
         float eps, T *__restrict__ y, float *__restrict__ mean, float *__restrict__ rstd)
{
    constexpr int RPB = norm_threads(TPR) / TPR;
    __shared__ float sm[32];
    after_previous();
    const int t = threadIdx.x % TPR;
    const unsigned step = gridDim.x * RPB;  // (rows are counted without a sign: the last one and a step may pass 2^31)
    const float inv = 1.0f / (float)N;
    const bool whole = on_32(gamma) && on_32(beta);
    unsigned r = blockIdx.x * RPB + threadIdx.x / TPR;
    Piece<T, VEC> next[CH];
    auto fetch = [&](unsigned row) {
        if (row < rows)
#pragma unroll
            for (int j = 0; j < CH; ++j)
                if ((j * TPR + t) * VEC < N) next[j].load(x + (size_t)row * N + (j * TPR + t) * VEC);
    };
    fetch(r);
    for (; r < rows; r += step) {
        const size_t at = (size_t)r * N;
        float v[CH][VEC];
        float sum[1] = {0.0f}, sq[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < CH; ++j)
            if ((j * TPR + t) * VEC < N) {
                next[j].get(v[j]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[0] += v[j][i];
            }
        fetch(r + step);  // on its way while this row is worked on
        row_join<false, TPR>(sum, sm);
        const float m = __fmul_rn(sum[0], inv);
#pragma unroll
        for (int j = 0; j < CH; ++j)
            if ((j * TPR + t) * VEC < N)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[j][i] -= m;
                    sq[0] = fmaf(v[j][i], v[j][i], sq[0]);
                }
        row_join<false, TPR>(sq, sm);
        const float s = 1.0f / sqrtf(sq[0] * inv + eps);
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
                if (gamma) load_f32<VEC>(gamma + c, whole, g);
                if (beta) load_f32<VEC>(beta + c, whole, b);
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
__global__ void __launch_bounds__(kWideThreads)
norm_fwd_wide(unsigned rows, int N, const T *__restrict__ x, const float *__restrict__ gamma,
              const float *__restrict__ beta, float eps, T *__restrict__ y, float *__restrict__ mean,
              float *__restrict__ rstd)
{
    __shared__ float sm[kWideThreads / 32];
    after_previous();
    const float inv = 1.0f / (float)N;
    for (unsigned r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *xr = x + (size_t)r * N;
        float sum = 0.0f, sq = 0.0f;
        for (int c = threadIdx.x; c < N; c += kWideThreads) sum += to_f32(xr[c]);
        const float m = __fmul_rn(row_sum<kWideThreads>(sum, sm), inv);
        for (int c = threadIdx.x; c < N; c += kWideThreads) {
            const float d = to_f32(xr[c]) - m;
            sq = fmaf(d, d, sq);
        }
        const float s = 1.0f / sqrtf(row_sum<kWideThreads>(sq, sm) * inv + eps);
        for (int c = threadIdx.x; c < N; c += kWideThreads)
            y[(size_t)r * N + c] = from_f32<T>(fmaf((to_f32(xr[c]) - m) * s, gamma ? gamma[c] : 1.0f, beta ? beta[c] : 0.0f));
        if (threadIdx.x == 0) {
            if (mean) mean[r] = m;
            if (rstd) rstd[r] = s;
        }
    }
}

// part [gridDim.x][2][N]: this CTA's sums of dy xh and dy over its rows. The pieces (of VEC > 1) of
// the next kAhead rows of a row's threads are on their way to shared memory while one is worked
// on, each copied by the thread that uses it; registers are left to the column sums. At 65536 x 1024
// bf16, forward and backward: 157 us with 8 warps an SM (the backward 106, 6.3 TB/s), 161 with three
// rows ahead and 166 with four (shared memory that L1 lacks), 166 with 12 warps; 192 with 12 warps
// and the next row in registers.
constexpr int kAhead = 2;
__host__ __device__ constexpr int norm_bwd_threads(int tpr, int elems) { return tpr == 32 && elems <= 16 ? 512 : 256; }
template <typename T>
__host__ __device__ constexpr size_t norm_row_bytes(int tpr, int vec, int ch)
{
    return vec > 1 ? (size_t)tpr * ch * vec * (4 + sizeof(T)) : 0;
}
template <typename T, int VEC, int CH, int TPR>
__global__ void __launch_bounds__(norm_bwd_threads(TPR, CH * VEC), TPR == 32 ? 1 : CH * VEC <= 16 ? 2 : 1)
norm_bwd(unsigned rows, int N, const float *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ gamma,
         const float *__restrict__ mean, const float *__restrict__ rstd, float *__restrict__ dx,
         float *__restrict__ part)
{
    constexpr int NT = norm_bwd_threads(TPR, CH * VEC), RPB = NT / TPR;
    constexpr size_t kRow = norm_row_bytes<T>(TPR, VEC, CH);
    __shared__ float sm[2 * 32];
    extern __shared__ __align__(16) uint8_t dyn[];  // the rows ahead; then the column sums [RPB][N]
    after_previous();
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const unsigned step = gridDim.x * RPB;
    const float inv = 1.0f / (float)N;
    const bool whole = on_32(gamma) && on_32(dx);
    float dg[CH][VEC], db[CH][VEC];
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) dg[j][i] = db[j][i] = 0.0f;
    // slot s of this thread: dy pieces at d(s) + j TPR VEC, x pieces at e(s) + j TPR VEC
    auto slot = [&](int s) { return dyn + ((size_t)s * RPB + sub) * kRow; };
    auto d_of = [&](int s) { return (float *)slot(s) + t * VEC; };
    auto x_of = [&](int s) { return (T *)(slot(s) + (size_t)TPR * CH * VEC * 4) + t * VEC; };
    auto fetch = [&](unsigned row, int s) {
        if constexpr (VEC > 1) {
            if (row < rows)
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    const int c = (j * TPR + t) * VEC;
                    if (c < N) {
                        const size_t o = (size_t)row * N + c;
#pragma unroll
                        for (int i = 0; i < VEC; i += 4) tc::cp_async16(tc::smem_u32(d_of(s) + j * TPR * VEC + i), dy + o + i, 16);
                        tc::cp_async16(tc::smem_u32(x_of(s) + j * TPR * VEC), x + o, 16);
                    }
                }
            tc::cp_async_commit();
        }
    };
    unsigned r = blockIdx.x * RPB + sub;
#pragma unroll
    for (int s = 0; s < kAhead; ++s) fetch(r + s * step, s);
    float next_m = r < rows ? mean[r] : 0.0f, next_rs = r < rows ? rstd[r] : 0.0f;
    for (int s = 0; r < rows; r += step, s = s + 1 == kAhead ? 0 : s + 1) {
        const size_t at = (size_t)r * N;
        const float m = next_m, rs = next_rs;
        if (r + step < rows) {
            next_m = mean[r + step];
            next_rs = rstd[r + step];
        }
        float a[CH][VEC], xh[CH][VEC];
        float sums[2] = {0.0f, 0.0f};  // of a and of a xh
        if constexpr (VEC > 1) tc::cp_async_wait<kAhead - 1>();
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + t) * VEC;
            if (c < N) {
                if constexpr (VEC > 1) {
                    load_vec<float, VEC>(d_of(s) + j * TPR * VEC, a[j]);
                    load_vec<T, VEC>(x_of(s) + j * TPR * VEC, xh[j]);
                } else {
                    load_vec<float, VEC>(dy + at + c, a[j]);
                    load_vec<T, VEC>(x + at + c, xh[j]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + t) * VEC;
            if (c < N) {
                float g[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] = 1.0f;
                if (gamma) load_f32<VEC>(gamma + c, whole, g);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    xh[j][i] = __fmul_rn(xh[j][i] - m, rs);
                    dg[j][i] = fmaf(a[j][i], xh[j][i], dg[j][i]);
                    db[j][i] += a[j][i];
                    a[j][i] = __fmul_rn(a[j][i], g[i]);
                    sums[0] += a[j][i];
                    sums[1] = fmaf(a[j][i], xh[j][i], sums[1]);
                }
            }
        }
        fetch(r + kAhead * step, s);  // into the slot just read
        if (dx) {
            row_join<false, TPR>(sums, sm);
            const float ma = __fmul_rn(sums[0], inv), mx = __fmul_rn(sums[1], inv);
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int c = (j * TPR + t) * VEC;
                if (c < N) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) a[j][i] = rs * (a[j][i] - ma - xh[j][i] * mx);
                    store_f32<VEC>(dx + at + c, whole, a[j]);
                }
            }
        }
    }
    if constexpr (VEC > 1) tc::cp_async_wait<0>();
    if (!part) return;
    float *out = part + (size_t)blockIdx.x * 2 * N, *cols = (float *)dyn;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (RPB > 1) __syncthreads();
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * TPR + t) * VEC;
            if (c < N) {
                float *to = RPB > 1 ? cols + (size_t)sub * N + c : out + (size_t)which * N + c;
                store_vec<float, VEC>(to, which ? db[j] : dg[j]);
            }
        }
        if constexpr (RPB > 1) {
            __syncthreads();
            for (int c = threadIdx.x; c < N; c += NT) {
                float acc = 0.0f;
#pragma unroll
                for (int w = 0; w < RPB; ++w) acc += cols[(size_t)w * N + c];
                out[(size_t)which * N + c] = acc;
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kWideThreads)
norm_bwd_wide(unsigned rows, int N, const float *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ gamma,
              const float *__restrict__ mean, const float *__restrict__ rstd, float *__restrict__ dx,
              float *__restrict__ part)
{
    __shared__ float sm[kWideThreads / 32];
    after_previous();
    const float inv = 1.0f / (float)N;
    float *out = part ? part + (size_t)blockIdx.x * 2 * N : nullptr;
    if (out)
        for (int c = threadIdx.x; c < 2 * N; c += kWideThreads) out[c] = 0.0f;
    __syncthreads();
    for (unsigned r = blockIdx.x; r < rows; r += gridDim.x) {
        const float *dr = dy + (size_t)r * N;
        const T *xr = x + (size_t)r * N;
        const float m = mean[r], s = rstd[r];
        float sa = 0.0f, sx = 0.0f;
        for (int c = threadIdx.x; c < N; c += kWideThreads) {
            const float a = dr[c] * (gamma ? gamma[c] : 1.0f);
            sa += a;
            sx = fmaf(a, (to_f32(xr[c]) - m) * s, sx);
        }
        const float ma = row_sum<kWideThreads>(sa, sm) * inv, mx = row_sum<kWideThreads>(sx, sm) * inv;
        for (int c = threadIdx.x; c < N; c += kWideThreads) {
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

// dgamma, dbeta = the parts' sums in a fixed order: warp w of a CTA adds parts w, w + 32, ... of 32
// columns, then the 32 sums are added in order. (Eight warps: 10 us for 608 parts of 400 columns.)
__global__ void __launch_bounds__(1024)
norm_reduce(const float *__restrict__ part, int n, int N, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    __shared__ float sm[32][33];
    after_previous();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const size_t c = blockIdx.x * (size_t)32 + lane, W = 2 * (size_t)N;
    float acc = 0.0f;
    if (c < W) {
#pragma unroll 10
        for (int s = w; s < n; s += 32) acc += part[(size_t)s * W + c];
    }
    sm[w][lane] = acc;
    __syncthreads();
    acc = warp_sum(sm[lane][w]);  // column w of the 32: a butterfly over the warps' sums
    const size_t cc = blockIdx.x * (size_t)32 + w;
    if (lane == 0 && cc < W) {
        if (cc < (size_t)N) {
            if (dgamma) dgamma[cc] = acc;
        } else if (dbeta) {
            dbeta[cc - N] = acc;
        }
    }
}

// How a call runs: elements of a piece, pieces a thread (0: the wide kernels), threads a row, CTAs.
struct NormPlan {
    int vec, ch, tpr, grid;
};
constexpr size_t kMostSumBytes = (size_t)4 << 30;  // of the CTAs' column sums: fewer CTAs from rows of 883011 on
inline size_t norm_sum_bytes(const stacklstm_op *op, const NormPlan &p) { return (size_t)p.grid * 2 * op->N * 4; }
NormPlan norm_plan(const stacklstm_op *op, int rows, bool bwd)
{
    const int vmax = op->dt == SL_BF16 ? 8 : 4, N = op->N;
    NormPlan p;
    p.vec = N % vmax == 0 ? vmax : 1;
    const int most = p.vec == 1 ? 16 : 4;
    p.tpr = ceil_div(N, p.vec * 32) <= (unsigned)most ? 32 : 256;
    const int n = (int)ceil_div(N, p.vec * p.tpr);
    p.ch = p.vec == 1 ? (n <= 4 ? 4 : n <= 16 ? 16 : 0) : n <= 1 ? 1 : n <= 2 ? 2 : n <= 4 ? 4 : 0;
    // (the backward: a CTA an SM of 8 or 16 rows, so that its column sums are few parts)
    const int per_sm = !p.ch ? 4 : bwd ? (p.tpr == 32 || p.ch * p.vec > 16 ? 1 : 2) : norm_ctas(p.tpr, p.ch * p.vec);
    const int rpb = !p.ch ? 1 : (bwd ? norm_bwd_threads(p.tpr, p.ch * p.vec) : norm_threads(p.tpr)) / p.tpr;
    p.grid = (int)std::min<size_t>(ceil_div((size_t)rows, (size_t)rpb), (size_t)op->num_sms * per_sm);
    if (bwd) p.grid = (int)std::min<size_t>(p.grid, std::max<size_t>(1, kMostSumBytes / ((size_t)N * 8)));
    return p;
}

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
};

template <typename T, int VEC, int CH, int TPR>
cudaError_t launch_norm(const NormCall &c, int grid)
{
    const int N = c.op->N;
    if (!c.dy) {
        return launch_after(norm_fwd<T, VEC, CH, TPR>, grid, norm_threads(TPR), 0, c.op->stream, c.rows, N, (const T *)c.x, c.gamma,
                            c.beta, c.eps, (T *)c.y, c.mean, c.rstd);
    } else {
        constexpr int NT = norm_bwd_threads(TPR, CH * VEC), RPB = NT / TPR;
        const size_t smem = std::max(kAhead * RPB * norm_row_bytes<T>(TPR, VEC, CH), RPB > 1 ? (size_t)RPB * N * 4 : 0);
        if (smem > 40 * 1024)
            if (cudaError_t e = smem_at_least((const void *)norm_bwd<T, VEC, CH, TPR>, smem)) return e;
        return launch_after(norm_bwd<T, VEC, CH, TPR>, grid, NT, smem, c.op->stream, c.rows, N, c.dy, (const T *)c.x, c.gamma,
                            (const float *)c.mean, (const float *)c.rstd, c.dx, c.part);
    }
}

template <typename T>
cudaError_t run_norm(const NormCall &c, const NormPlan &p)
{
    constexpr int V = 16 / (int)sizeof(T);
#define SL_NORM(v, n, t) \
    if (p.vec == v && p.ch == n && p.tpr == t) return launch_norm<T, v, n, t>(c, p.grid);
    SL_NORM(V, 1, 32) SL_NORM(V, 2, 32) SL_NORM(V, 4, 32) SL_NORM(V, 1, 256) SL_NORM(V, 2, 256) SL_NORM(V, 4, 256)
    SL_NORM(1, 4, 32) SL_NORM(1, 16, 32) SL_NORM(1, 4, 256) SL_NORM(1, 16, 256)
#undef SL_NORM
    if (!c.dy)
        return launch_after(norm_fwd_wide<T>, p.grid, kWideThreads, 0, c.op->stream, c.rows, c.op->N, (const T *)c.x, c.gamma, c.beta,
                            c.eps, (T *)c.y, c.mean, c.rstd);
    return launch_after(norm_bwd_wide<T>, p.grid, kWideThreads, 0, c.op->stream, c.rows, c.op->N, c.dy, (const T *)c.x, c.gamma,
                        (const float *)c.mean, (const float *)c.rstd, c.dx, c.part);
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
    // the column sums of a backward's CTAs: 10 MB at most; for the wide kernels, where they are gigabytes,
    // the first backward that wants them allocates them
    const NormPlan p = norm_plan(op, R, true);
    if (p.ch && op_workspace(op, 0, norm_sum_bytes(op, p)) != cudaSuccess) {
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
    const NormPlan p = norm_plan(op, rows, false);
    const cudaError_t e = op->dt == SL_BF16 ? run_norm<__nv_bfloat16>(c, p) : run_norm<float>(c, p);
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
    const NormPlan p = norm_plan(op, rows, true);
    if (sums && (e = op_workspace(op, 0, norm_sum_bytes(op, p)))) return op_cuda(op, e, "stacklstm_norm_backward");
    c.part = sums ? (float *)op->ws[0] : nullptr;
    e = op->dt == SL_BF16 ? run_norm<__nv_bfloat16>(c, p) : run_norm<float>(c, p);
    if (!e && sums)
        e = launch_after(norm_reduce, ceil_div(2 * (size_t)op->N, 32), 1024, 0, op->stream, (const float *)op->ws[0], p.grid, op->N,
                         dgamma, dbeta);
    return e ? op_cuda(op, e, "stacklstm_norm_backward") : SL_OK;
}

}  // extern "C"
