// distill.cu -- distillation from a teacher's top logits: loss and gradient in one pass, and its
// C ABI (include/stacklstm.h, stacklstm_distill_*).
//
// Row r has V logits z and up to k teacher entries (class i_j, logit t_j). With q the softmax of
// t / tau over the entries present, p = softmax(z / tau) and P = softmax(z),
//   loss = scale [ alpha tau^2 sum_j q_j (ln q_j - ln p_{i_j}) + (1 - alpha) (-ln P_gold) ]
//   dz_v = scale [ alpha tau (p_v - sum_{j: i_j = v} q_j) + (1 - alpha) (P_v - [v = gold]) ],
// each term only where the row has a teacher (a gold class).
// Bound by HBM: z is read once (into the registers of the row's threads, where the widths allow),
// dz is written once. Both softmaxes share the maximum of z; the sums are fp32.
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

// NP pieces a thread in registers (0: read again in each pass); RPC rows a CTA.
template <typename T, int TPR, int NP>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR)
distill_rows(const DistillArgs a)
{
    constexpr int E = RowVec<T>::E, RPC = TPR == 32 ? 8 : 1;
    __shared__ float sm[kRowThreads / 32];
    extern __shared__ uint8_t dyn[];
    const int sub = TPR == 32 ? threadIdx.x / 32 : 0, t = threadIdx.x % TPR;
    const int r = blockIdx.x * RPC + sub;
    if (r >= a.rows) return;  // (TPR = 32: no barrier of the CTA below)
    int *ci = (int *)dyn + (size_t)sub * (a.k + 1);                           // classes of the entries
    float *cw = (float *)(dyn + (size_t)RPC * (a.k + 1) * 4) + (size_t)sub * (a.k + 1);  // their weights in the gradient
    auto sync = [] {
        if constexpr (TPR == 32)
            __syncwarp();
        else
            __syncthreads();
    };
    const T *z = (const T *)a.z;
    const RowVec<T> row(r, a.V, a.rows);
    const int n = row.pieces();
    float v[NP > 0 ? NP : 1][E];
    float m = -INFINITY;
    if constexpr (NP > 0) {
#pragma unroll
        for (int j = 0; j < NP; ++j)
            if (j * TPR + t < n) row.load(z, j * TPR + t, v[j]);
#pragma unroll
        for (int j = 0; j < NP; ++j)
            if (j * TPR + t < n)
#pragma unroll
                for (int i = 0; i < E; ++i) m = max_nan(m, v[j][i]);
    } else {
        for (int p = t; p < n; p += TPR) {
            row.load(z, p, v[0]);
#pragma unroll
            for (int i = 0; i < E; ++i) m = max_nan(m, v[0][i]);
        }
    }
    // the teacher, by the row's first warp (each warp when it is the row)
    float tmax = -INFINITY, tsum = 0.0f;
    for (int j = t; j < a.k; j += TPR) {
        int c = a.t_idx[(size_t)r * a.k + j];
        float l = a.t_logit[(size_t)r * a.k + j];
        if (c < -1 || c >= a.V) {
            atomicCAS(a.err, 0, (int)SL_ERR_ARG);  // the entry is skipped
            c = -1;
        }
        if (l == -INFINITY) c = -1;
        ci[j] = c;
        cw[j] = l;
    }
    sync();
    for (int j = (int)(threadIdx.x & 31); j < a.k; j += 32)
        if (ci[j] >= 0) tmax = fmaxf(tmax, cw[j]);
    tmax = warp_max(tmax);
    for (int j = (int)(threadIdx.x & 31); j < a.k; j += 32)
        if (ci[j] >= 0) tsum += expf((cw[j] - tmax) / a.tau);
    tsum = warp_sum(tsum);
    int gold = a.gold ? a.gold[r] : -1;
    if (gold < -1 || gold >= a.V) {
        if (t == 0) atomicCAS(a.err, 0, (int)SL_ERR_ARG);
        gold = -1;
    }
    m = row_max<TPR>(m, sm);
    const bool some = m > -INFINITY || isnan(m);
    // (a teacher whose logits are all -inf, or absent, has tsum = 0)
    const bool soft = some && a.alpha > 0.0f && tsum != 0.0f, hard = some && a.alpha < 1.0f && gold >= 0;
    const float k2 = kLog2e / a.tau;
    float st = 0.0f, s1 = 0.0f;
    auto add = [&](const float (&w)[E]) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float d = w[i] - m;
            if (soft) st += exp2_hw(d * k2);
            if (hard) s1 += exp2_hw(d * kLog2e);
        }
    };
    if (soft || hard) {
        if constexpr (NP > 0) {
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if (j * TPR + t < n) add(v[j]);
        } else {
            for (int p = t; p < n; p += TPR) {
                row.load(z, p, v[0]);
                add(v[0]);
            }
        }
    }
    st = row_sum<TPR>(st, sm);
    s1 = row_sum<TPR>(s1, sm);
    const float lse_t = logf(st), lse_1 = logf(s1);  // of (z - m) / tau and z - m
    const float ct = soft ? a.scale * a.alpha * a.tau : 0.0f, c1 = hard ? a.scale * (1.0f - a.alpha) : 0.0f;
    const float wt = soft ? ct / st : 0.0f, w1 = hard ? c1 / s1 : 0.0f;
    auto grad = [&](float zv) {
        const float d = zv - m;
        float g = 0.0f;
        if (soft) g = wt * exp2_hw(d * k2);
        if (hard) g = fmaf(w1, exp2_hw(d * kLog2e), g);
        return g;
    };
    if (a.dz) {
        auto put = [&](int p, const float (&w)[E]) {
            float g[E];
#pragma unroll
            for (int i = 0; i < E; ++i) g[i] = grad(w[i]);
            row.store_f32(a.dz, p, g);
        };
        if constexpr (NP > 0) {
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if (j * TPR + t < n) put(j * TPR + t, v[j]);
        } else {
            for (int p = t; p < n; p += TPR) {
                row.load(z, p, v[0]);
                put(p, v[0]);
            }
        }
    }
    // the loss, and the entries' weights; entry k is the gold class
    float loss = 0.0f;
    if (soft)
        for (int j = (int)(threadIdx.x & 31); j < a.k; j += 32)
            if (ci[j] >= 0) {
                const float l = (cw[j] - tmax) / a.tau, q = expf(l) / tsum;
                if (q > 0.0f) loss += q * ((l - logf(tsum)) - ((to_f32(z[row.first + ci[j]]) - m) / a.tau - lse_t));
            }
    loss = warp_sum(loss) * a.alpha * a.tau * a.tau;
    if (hard) loss += (1.0f - a.alpha) * (lse_1 - (to_f32(z[row.first + gold]) - m));
    if (t == 0 && a.loss) a.loss[r] = a.scale * loss;
    if (!a.dz) return;
    sync();
    for (int j = t; j <= a.k; j += TPR) {
        if (j == a.k) {
            ci[j] = hard ? gold : -1;
            cw[j] = c1;
        } else if (ci[j] >= 0) {
            if (soft)
                cw[j] = ct * (expf((cw[j] - tmax) / a.tau) / tsum);
            else
                ci[j] = -1;
        }
    }
    sync();
    for (int j = t; j <= a.k; j += TPR) {
        const int c = ci[j];
        if (c < 0) continue;
        bool first = true;
        for (int i = 0; i < j; ++i) first = first && ci[i] != c;
        if (!first) continue;
        float w = 0.0f;
        for (int i = j; i <= a.k; ++i)
            if (ci[i] == c) w += cw[i];
        a.dz[row.first + c] = grad(to_f32(z[row.first + c])) - w;
    }
}

template <typename T>
cudaError_t launch_distill(const DistillArgs &a, cudaStream_t st)
{
    int tpr, np;
    row_plan<T>(a.V, &tpr, &np);
    const int rpc = tpr == 32 ? 8 : 1;
    const unsigned grid = ceil_div(a.rows, rpc);
    const size_t smem = (size_t)rpc * (a.k + 1) * 8;
#define SL_DIST(t, n) \
    if (tpr == t && np == n) distill_rows<T, t, n><<<grid, t == 32 ? 256 : t, smem, st>>>(a);
    SL_DIST(32, 1) SL_DIST(32, 2) SL_DIST(32, 4)
    SL_DIST(kRowThreads, 0) SL_DIST(kRowThreads, 1) SL_DIST(kRowThreads, 2) SL_DIST(kRowThreads, 4)
    SL_DIST(kRowThreads, 8) SL_DIST(kRowThreads, 16)
#undef SL_DIST
    return cudaGetLastError();
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
    const cudaError_t e = op->dt == SL_BF16 ? launch_distill<__nv_bfloat16>(a, op->stream) : launch_distill<float>(a, op->stream);
    return e ? op_cuda(op, e, "stacklstm_distill_run") : SL_OK;
}

}  // extern "C"
