// distill.cu -- distillation from a teacher's top logits: loss and gradient in one pass, and its
// C ABI (include/stacklstm.h, stacklstm_distill_*).
//
// Row r has V logits z and up to k teacher entries (class i_j, logit t_j). With q the softmax of
// t / tau over the entries present, p = softmax(z / tau) and P = softmax(z),
//   loss = scale [ alpha tau^2 sum_j q_j (ln q_j - ln p_{i_j}) + (1 - alpha) (-ln P_gold) ]
//   dz_v = scale [ alpha tau (p_v - sum_{j: i_j = v} q_j) + (1 - alpha) (P_v - [v = gold]) ],
// each term only where the row has a teacher (a gold class).
// Bound by HBM: z is read from it once (and again from the caches where a row is wide), dz is
// written once. Both softmaxes share the maximum of z; the sums are fp32.
// The few classes of the teacher and the gold class are written once more after the row's dense
// gradient: the first entry of each class takes the sum of the class's weights in entry order, so
// that repeated classes need no atomics and the result does not depend on timing.
#include "rowvec.cuh"

namespace sl {
namespace {

constexpr int kMaxTeacher = 256;

struct DistillArgs {
    int rows, V, k;
    const void *z;
    const int32_t *t_idx;
    const float *t_logit;
    const int32_t *gold;
    float tau, alpha, scale;
    float *loss, *dz;
    int32_t *err;
};

// With l_j = (t_j - max t) / tau, w_j = exp(l_j) and x_v = z_v - max z, a row needs four sums:
// sum_j w_j, sum_j w_j (l_j - x_{i_j} / tau), sum_v exp(x_v / tau) and sum_v exp(x_v).

// An entry's place in a row: its class (-1: none), teacher's logit (later its weight), its class's z.
struct Entries {
    int *c;
    float *w, *z;
};

// Entry j of row r, checked.
template <typename T>
__device__ __forceinline__ float read_entry(const DistillArgs &a, const Entries &e, size_t r, const T *zr, int j)
{
    int c = a.t_idx[r * a.k + j];
    const float l = a.t_logit[r * a.k + j];
    if (c < -1 || c >= a.V) {
        atomicCAS(a.err, 0, (int)SL_ERR_ARG);  // the entry is skipped
        c = -1;
    }
    if (l == -INFINITY) c = -1;
    e.c[j] = c;
    e.w[j] = l;
    if (c < 0) return -INFINITY;
    e.z[j] = to_f32(zr[c]);
    return l;
}
// The gold class of row r, checked (lead: the thread that reports).
__device__ __forceinline__ int read_gold(const DistillArgs &a, size_t r, bool lead)
{
    int gold = a.gold ? a.gold[r] : -1;
    if (gold < -1 || gold >= a.V) {
        if (lead) atomicCAS(a.err, 0, (int)SL_ERR_ARG);
        gold = -1;
    }
    return gold;
}
// Entry j's share of the two sums over the entries; its logit becomes its weight before the sum's
// division.
__device__ __forceinline__ void add_entry(const Entries &e, int j, float top, float m, float rtau, float &s0, float &s1)
{
    if (e.c[j] < 0) return;
    const float l = (e.w[j] - top) * rtau, w = expf(l);
    s0 += w;
    if (w > 0.0f)
        s1 += w * (l - (e.z[j] - m) * rtau);  // (weight 0 on a class of -inf is 0)
    else if (isnan(w))
        s1 = w;
    e.w[j] = w;
}

// Two neighbours at a time, each rounded as one alone: the differences from m, and 2^(d k). (The
// logits less m times k as one operation, k z - k m, would not hold for masks of the type's lowest
// value, where k m overflows.)
__device__ __forceinline__ float2 less2(float a, float b, float m) { return __fadd2_rn(make_float2(a, b), make_float2(-m, -m)); }
__device__ __forceinline__ float2 exp2_2(float2 d, float k)
{
    const float2 x = __fmul2_rn(d, make_float2(k, k));
    return make_float2(exp2_hw(x.x), exp2_hw(x.y));
}

// What a row's outputs are made of.
struct Row {
    float m, wt, w1;   // gradient: wt exp((z - m) / tau) + w1 exp(z - m)
    float ct, c1;      // the weights of the teacher's entries (over their sum) and of the gold class
    bool soft, hard;
    float k2;          // log2(e) / tau
    __device__ __forceinline__ Row(const DistillArgs &a, float m_, float top, int gold) : m(m_), k2(kLog2e / a.tau)
    {
        const bool some = m > -INFINITY || isnan(m), taught = top > -INFINITY || isnan(top);
        soft = some && taught && a.alpha > 0.0f;
        hard = some && gold >= 0 && a.alpha < 1.0f;
        ct = soft ? a.scale * a.alpha * a.tau : 0.0f;
        c1 = hard ? a.scale * (1.0f - a.alpha) : 0.0f;
    }
    __device__ __forceinline__ void sums(const float (&s)[4])
    {
        wt = soft ? ct / s[2] : 0.0f;
        w1 = hard ? c1 / s[3] : 0.0f;
    }
    __device__ __forceinline__ float grad(float z) const
    {
        const float d = z - m;
        float g = 0.0f;
        if (soft) g = wt * exp2_hw(d * k2);
        if (hard) g = fmaf(w1, exp2_hw(d * kLog2e), g);
        return g;
    }
    __device__ __forceinline__ float loss(const DistillArgs &a, const float (&s)[4], float zgold) const
    {
        float l = 0.0f;
        if (soft) l = a.alpha * a.tau * a.tau * (s[1] / s[0] - logf(s[0]) + logf(s[2]));
        if (hard) l += (1.0f - a.alpha) * (logf(s[3]) - (zgold - m));
        return a.scale * l;
    }
    // the gradient of a piece
    template <int E>
    __device__ __forceinline__ void grads(const float (&v)[E], float (&g)[E]) const
    {
        if (soft && hard) {
#pragma unroll
            for (int i = 0; i < E; i += 2) {
                const float2 d = less2(v[i], v[i + 1], m);
                const float2 x = __ffma2_rn(make_float2(w1, w1), exp2_2(d, kLog2e),
                                            __fmul2_rn(make_float2(wt, wt), exp2_2(d, k2)));
                g[i] = x.x;
                g[i + 1] = x.y;
            }
        } else {
            const float kk = soft ? k2 : kLog2e, w = soft ? wt : w1;
#pragma unroll
            for (int i = 0; i < E; ++i) g[i] = soft || hard ? w * exp2_hw((v[i] - m) * kk) : 0.0f;
        }
    }
    // entry j's weight in the gradient, or that it has none
    __device__ __forceinline__ void weigh(const Entries &e, int j, float s0) const
    {
        if (e.c[j] < 0) return;
        if (soft)
            e.w[j] = ct * (e.w[j] / s0);
        else
            e.c[j] = -1;
    }
    // entry k: the gold class
    __device__ __forceinline__ void gold_entry(const Entries &e, int k, int gold, float zgold) const
    {
        e.c[k] = hard ? gold : -1;
        e.w[k] = c1;
        e.z[k] = zgold;
    }
};

// Rows of up to 4 pieces a lane: TPR lanes (8 or 32) to a row, NP pieces a lane in registers, as
// they lie in memory. A call of 11840 x 83 fp32 with 8 entries a row is 6.4 us, bound by the call.
template <typename T, int TPR, int NP>
__global__ void __launch_bounds__(256, 5)
distill_narrow(const __grid_constant__ DistillArgs a)
{
    constexpr int E = RowVec<T>::E, RPC = 256 / TPR;
    extern __shared__ __align__(16) uint8_t dyn[];
    after_previous();
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR, k1 = a.k + 1;
    const Entries e = {(int *)dyn + (size_t)sub * k1, (float *)(dyn + (size_t)RPC * k1 * 4) + (size_t)sub * k1,
                       (float *)(dyn + (size_t)RPC * k1 * 8) + (size_t)sub * k1};
    const size_t r = (size_t)blockIdx.x * RPC + sub;
    const bool here = r < (size_t)a.rows;  // (lanes of a row past the end stay for the joins)
    const T *z = (const T *)a.z;
    const RowVec<T> row(r, a.V);
    const T *zr = z + row.first();
    const int n = here ? row.pieces() : 0, k = here ? a.k : 0;
    uint4 q[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j)
        if (j * TPR + t < n) q[j] = row.load(z, j * TPR + t);
    auto each = [&](auto f) {  // f(piece, its elements) over this lane's pieces
#pragma unroll
        for (int j = 0; j < NP; ++j)
            if (j * TPR + t < n) {
                float v[E];
                unpack<T>(q[j], v);
                f(j * TPR + t, v);
            }
    };
    float top[2] = {-INFINITY, -INFINITY};  // of z, of the teacher's logits
    for (int j = t; j < k; j += TPR) top[1] = max_nan(top[1], read_entry(a, e, r, zr, j));
    const int gold = here ? read_gold(a, r, t == 0) : -1;
    const float zgold = t == 0 && gold >= 0 ? to_f32(zr[gold]) : 0.0f;  // (lane 0 uses it)
#pragma unroll
    for (int j = 0; j < NP; ++j)
        if (j * TPR + t < n) top[0] = max_nan(top[0], piece_max<T, true>(q[j]));
    lanes_join<true, TPR>(top);
    Row w(a, top[0], top[1], gold);
    const float rtau = 1.0f / a.tau;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (w.soft)
        for (int j = t; j < k; j += TPR) add_entry(e, j, top[1], w.m, rtau, s[0], s[1]);
    if (w.soft || w.hard)
        each([&](int, const float (&v)[E]) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float d = v[i] - w.m;
                if (w.soft) s[2] += exp2_hw(d * w.k2);
                if (w.hard) s[3] += exp2_hw(d * kLog2e);
            }
        });
    lanes_join<false, TPR>(s);
    w.sums(s);
    if (t == 0 && here && a.loss) a.loss[r] = w.loss(a, s, zgold);
    if (!a.dz) return;
    const bool aligned = on_32(a.dz);
    for (int j = t; j < k; j += TPR) w.weigh(e, j, s[0]);
    if (t == 0) w.gold_entry(e, a.k, gold, zgold);
    each([&](int p, const float (&v)[E]) {
        float g[E];
        w.grads(v, g);
        row.store_f32(a.dz, aligned, p, g);
    });
    __syncwarp();  // the row's gradient, and its entries
    if (!here) return;
    for (int j = t; j <= a.k; j += TPR) {
        const int c = e.c[j];
        if (c < 0) continue;
        bool first = true;
        float wj = e.w[j];
        for (int i = 0; i <= a.k; ++i)
            if (e.c[i] == c) {
                if (i < j) first = false;
                if (i > j) wj += e.w[i];
            }
        if (first) a.dz[row.first() + c] = w.grad(e.z[j]) - wj;
    }
}

// Wider rows: a CTA of TPR threads a row, the row read twice, the second time from the caches. A
// thread keeps its own maximum and the sums against it, so that the first reading is one pass; 1536
// threads an SM hide one another's latencies. At 4096 x 32003 bf16: 153 us with 512 threads a row
// (5.1 TB/s), two elements at a time; one at a time 156 (the warps' issue is what bounds it next to
// HBM). With one at a time everywhere: 159 with 512 threads a row, 164 with 256, 186 with 128; 182
// with the row held in the registers of 512 threads, two CTAs an SM, and no less with the next row on
// its way to shared memory: the barriers and the entries' part of each row were not hidden.
template <typename T, int TPR>
__global__ void __launch_bounds__(TPR, 1536 / TPR)
distill_wide(const __grid_constant__ DistillArgs a)
{
    constexpr int E = RowVec<T>::E, NW = TPR / 32;
    __shared__ float sm_max[2 * 32], sm_sum[4 * 32];
    __shared__ int ec[kMaxTeacher + 1];
    __shared__ float ew[kMaxTeacher + 1], ez[kMaxTeacher + 1];
    after_previous();
    const Entries e = {ec, ew, ez};
    const int t = threadIdx.x, lane = t & 31;
    const size_t r = blockIdx.x;
    const T *z = (const T *)a.z;
    const RowVec<T> row(r, a.V);
    const T *zr = z + row.first();
    const int n = row.pieces();
    const float k2 = kLog2e / a.tau;
    const bool want2 = a.alpha > 0.0f, want1 = a.alpha < 1.0f;
    float top[2] = {-INFINITY, -INFINITY};
    for (int j = t; j < a.k; j += TPR) top[1] = max_nan(top[1], read_entry(a, e, r, zr, j));
    const int gold = read_gold(a, r, t == 0);
    const float zgold = t == 0 && gold >= 0 ? to_f32(zr[gold]) : 0.0f;
    // the first pass, four pieces in flight; m: this thread's maximum, s2 and s1 against it
    // for even and odd elements apart
    float m = -INFINITY;
    float2 s2 = {0.0f, 0.0f}, s1 = {0.0f, 0.0f};
    auto add = [&](const uint4 &q) {
        const float pm = piece_max<T, true>(q);
        if (!(pm <= m)) {  // a new maximum (or NaN)
            const float d = m - pm;  // (-inf at first: the sums are 0)
            const float c2 = exp2_hw(d * k2), c1 = exp2_hw(d * kLog2e);
            s2 = __fmul2_rn(s2, make_float2(c2, c2));
            s1 = __fmul2_rn(s1, make_float2(c1, c1));
            m = max_nan(m, pm);  // (a NaN stays, whatever follows it)
        }
        if (m == -INFINITY) return;  // nothing yet
        float v[E];
        unpack<T>(q, v);
        if (want2 && want1) {
#pragma unroll
            for (int i = 0; i < E; i += 2) {
                const float2 d = less2(v[i], v[i + 1], m);
                s2 = __fadd2_rn(s2, exp2_2(d, k2));
                s1 = __fadd2_rn(s1, exp2_2(d, kLog2e));
            }
        } else {
            const float kk = want2 ? k2 : kLog2e;
            float2 s = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < E; i += 2) s = __fadd2_rn(s, exp2_2(less2(v[i], v[i + 1], m), kk));
            if (want2) s2 = __fadd2_rn(s2, s);
            else s1 = __fadd2_rn(s1, s);
        }
    };
    for (int p = t; p < n; p += 4 * TPR) {
        uint4 q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (p + u * TPR < n) q[u] = row.load(z, p + u * TPR);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (p + u * TPR < n) add(q[u]);
    }
    top[0] = m;
    row_join<true, TPR, true>(top, sm_max);
    Row w(a, top[0], top[1], gold);
    const float rtau = 1.0f / a.tau;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (m > -INFINITY || isnan(m)) {  // this thread's sums against the row's maximum
        s[2] = (s2.x + s2.y) * exp2_hw((m - w.m) * k2);
        s[3] = (s1.x + s1.y) * exp2_hw((m - w.m) * kLog2e);
    }
    if (w.soft)
        for (int j = t; j < a.k; j += TPR) add_entry(e, j, top[1], w.m, rtau, s[0], s[1]);
    row_join<false, TPR, true>(s, sm_sum);
    w.sums(s);
    if (t == 0 && a.loss) a.loss[r] = w.loss(a, s, zgold);
    if (!a.dz) return;
    const bool aligned = on_32(a.dz);
    for (int j = t; j < a.k; j += TPR) w.weigh(e, j, s[0]);
    if (t == 0) w.gold_entry(e, a.k, gold, zgold);
    for (int p = t; p < n; p += 2 * TPR) {
        uint4 q[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (p + u * TPR < n) q[u] = row.load(z, p + u * TPR);
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (p + u * TPR < n) {
                float v[E], g[E];
                unpack<T>(q[u], v);
                w.grads(v, g);
                row.store_f32(a.dz, aligned, p + u * TPR, g);
            }
    }
    __syncthreads();  // the row's gradient, and its entries
    for (int j = t / 32; j <= a.k; j += NW) {  // a warp an entry
        const int c = e.c[j];
        if (c < 0) continue;
        bool earlier = false;
        float wj = 0.0f;
        for (int i = lane; i <= a.k; i += 32)
            if (e.c[i] == c) {
                earlier = earlier || i < j;
                wj += e.w[i];
            }
        if (__any_sync(0xffffffffu, earlier)) continue;
        wj = warp_sum(wj);
        if (lane == 0) a.dz[row.first() + c] = w.grad(e.z[j]) - wj;
    }
}

template <typename T>
cudaError_t launch_distill(const stacklstm_op *op, const DistillArgs &a)
{
    int tpr, np;
    row_plan<T>(a.V, &tpr, &np);
    if (tpr <= 32) {
        const unsigned grid = ceil_div(a.rows, 256 / tpr);
        const size_t smem = (size_t)(256 / tpr) * (a.k + 1) * 12;  // (at most 99 KB)
        auto launch = [&](auto kernel) {
            if (smem > 48 * 1024)
                if (cudaError_t e = smem_at_least((const void *)kernel, smem)) return e;
            return launch_after(kernel, grid, 256, smem, op->stream, a);
        };
        return tpr == 8 ? launch(np == 1 ? distill_narrow<T, 8, 1> : np == 2 ? distill_narrow<T, 8, 2> : distill_narrow<T, 8, 4>)
                        : launch(np <= 2 ? distill_narrow<T, 32, 2> : distill_narrow<T, 32, 4>);
    }
    return tpr == 128 ? launch_after(distill_wide<T, 128>, a.rows, 128, 0, op->stream, a)
                      : launch_after(distill_wide<T, 512>, a.rows, 512, 0, op->stream, a);
}

}  // namespace
}  // namespace sl

using namespace sl;

extern "C" {

sl_status stacklstm_distill_create(stacklstm_op_t *out, int R, int V, int k, sl_dtype dtype, int device, void *stream)
{
    if (!out) return SL_ERR_ARG;
    *out = nullptr;
    if (R < 1 || V < 1 || k < 1 || (dtype != SL_FP32 && dtype != SL_BF16)) return SL_ERR_ARG;
    if (k > kMaxTeacher || V > (1 << 30)) return SL_ERR_UNSUPPORTED;
    sl_status st;
    stacklstm_op *op = op_new(SL_OP_DISTILL, dtype, device, stream, &st);
    if (!op) return st;
    op->R = R;
    op->V = V;
    op->k = k;
    *out = op;
    return SL_OK;
}

sl_status stacklstm_distill_run(stacklstm_op_t op, int rows, const void *logits, const int32_t *t_idx,
                                const float *t_logit, const int32_t *gold, float tau, float alpha, float scale,
                                float *loss_rows, float *dlogits)
{
    if (!op || op->kind != SL_OP_DISTILL) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (rows < 0 || rows > op->R) return op_fail(op, SL_ERR_ARG, "rows outside 0 .. R");
    if (!(tau > 0.0f) || !(tau < INFINITY)) return op_fail(op, SL_ERR_ARG, "tau must be positive and finite");
    if (!(alpha >= 0.0f && alpha <= 1.0f)) return op_fail(op, SL_ERR_ARG, "alpha outside 0 .. 1");
    if (rows == 0) return SL_OK;
    if (const char *m = check_pointers({logits, t_idx, t_logit}, {gold, loss_rows, dlogits}))
        return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    DistillArgs a;
    a.rows = rows; a.V = op->V; a.k = op->k; a.z = logits; a.t_idx = t_idx; a.t_logit = t_logit; a.gold = gold;
    a.tau = tau; a.alpha = alpha; a.scale = scale; a.loss = loss_rows; a.dz = dlogits; a.err = op->err;
    const cudaError_t e = op->dt == SL_BF16 ? launch_distill<__nv_bfloat16>(op, a) : launch_distill<float>(op, a);
    return e ? op_cuda(op, e, "stacklstm_distill_run") : SL_OK;
}

}  // extern "C"
