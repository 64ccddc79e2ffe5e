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
#include "tc.cuh"

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

// Threads TPR to a row (8 or 32 lanes: several rows a warp or CTA; else the whole CTA), NP pieces a
// thread in registers, as they lie in memory (0: read again in each pass). A CTA takes rows
// gridDim.x rows_per_cta apart; where a row is the CTA's, the pieces and the teacher's entries of
// its next one are copied to shared memory while one is worked on, each by the thread that uses it
// (4096 x 32003 bf16: 202 us without).
// With l_j = (t_j - max t) / tau, w_j = exp(l_j) and x_v = z_v - max z, four sums are joined at
// once: sum_j w_j, sum_j w_j (l_j - x_{i_j} / tau), sum_v exp(x_v / tau), sum_v exp(x_v).
template <typename T, int TPR, int NP>
__global__ void __launch_bounds__(row_cta(TPR), row_ctas_per_sm(TPR))
distill_rows(const __grid_constant__ DistillArgs a)
{
    constexpr int E = RowVec<T>::E, RPC = rows_per_cta(TPR);
    constexpr bool AHEAD = TPR > 32 && NP > 0;
    __shared__ float sm[4 * 32];
    extern __shared__ __align__(16) uint8_t dyn[];
    const int sub = TPR <= 32 ? threadIdx.x / TPR : 0, t = threadIdx.x % TPR, k1 = a.k + 1;
    uint4 *ahead = (uint4 *)dyn + threadIdx.x;  // piece j at ahead[j TPR]
    uint8_t *dyn2 = dyn + (AHEAD ? (size_t)TPR * NP * 16 : 0);
    int *ci = (int *)dyn2 + (size_t)sub * k1;                          // classes of the entries
    float *cw = (float *)(dyn2 + (size_t)RPC * k1 * 4) + (size_t)sub * k1;  // their logits, then weights
    float *cz = (float *)(dyn2 + (size_t)RPC * k1 * 8) + (size_t)sub * k1;  // z - max z of their classes
    auto sync = [] {
        if constexpr (TPR <= 32)
            __syncwarp();
        else
            __syncthreads();
    };
    const T *z = (const T *)a.z;
    const int step = gridDim.x * RPC;
    const bool aligned = on_32(a.dz);
    // the next row's pieces (whole ones) on their way, and its entry of this thread and gold class
    int next_c = -1, next_gold = -1;
    float next_l = 0.0f;
    auto fetch = [&](int row_i) {
        if constexpr (AHEAD) {
            if (row_i < a.rows) {
                const RowVec<T> row(row_i, a.V);
                const int n = row.pieces();
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    const int p = j * TPR + t;
                    if (p < n && row.whole(p))
                        tc::cp_async16(tc::smem_u32(ahead + j * TPR), z + row.at + (size_t)p * E, 16);
                }
                if (t < a.k) {
                    next_c = a.t_idx[(size_t)row_i * a.k + t];
                    next_l = a.t_logit[(size_t)row_i * a.k + t];
                }
                next_gold = a.gold ? a.gold[row_i] : -1;
            }
            tc::cp_async_commit();
        }
    };
    int r0 = blockIdx.x * RPC;
    fetch(r0);
    for (; r0 < a.rows; r0 += step) {
        const int r = r0 + sub;
        const bool here = r < a.rows;  // (lanes of a row past the end stay for the joins)
        const RowVec<T> row(r, a.V);
        const T *zr = z + row.first();
        const int n = here ? row.pieces() : 0, k = here ? a.k : 0;
        uint4 q[NP > 0 ? NP : 1];
        if constexpr (AHEAD) tc::cp_async_wait<0>();
        if constexpr (NP > 0) {
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int p = j * TPR + t;
                if (p < n) q[j] = AHEAD && row.whole(p) ? ahead[j * TPR] : row.load(z, p);
            }
        }
        // f(piece, its elements) over this thread's pieces
        auto each = [&](auto f) {
            if constexpr (NP > 0) {
#pragma unroll
                for (int j = 0; j < NP; ++j)
                    if (j * TPR + t < n) {
                        float v[E];
                        unpack<T>(q[j], v);
                        f(j * TPR + t, v);
                    }
            } else {
                for (int p = t; p < n; p += TPR) {
                    float v[E];
                    unpack<T>(row.load(z, p), v);
                    f(p, v);
                }
            }
        };
        float top[2] = {-INFINITY, -INFINITY};  // of z, of the teacher's logits
        int gold = AHEAD ? next_gold : here && a.gold ? a.gold[r] : -1;
        for (int j = t; j < k; j += TPR) {
            int c = AHEAD && j == t ? next_c : a.t_idx[(size_t)r * a.k + j];
            const float l = AHEAD && j == t ? next_l : a.t_logit[(size_t)r * a.k + j];
            if (c < -1 || c >= a.V) {
                atomicCAS(a.err, 0, (int)SL_ERR_ARG);  // the entry is skipped
                c = -1;
            }
            if (l == -INFINITY) c = -1;
            ci[j] = c;
            cw[j] = l;
            if (c >= 0) {
                cz[j] = to_f32(zr[c]);
                top[1] = max_nan(top[1], l);
            }
        }
        if (gold < -1 || gold >= a.V) {
            if (t == 0) atomicCAS(a.err, 0, (int)SL_ERR_ARG);
            gold = -1;
        }
        const float zgold = t == 0 && gold >= 0 ? to_f32(zr[gold]) : 0.0f;  // (thread 0 uses it)
        if constexpr (NP > 0) {
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if (j * TPR + t < n) top[0] = max_nan(top[0], piece_max<T, true>(q[j]));
        } else {
            for (int p = t; p < n; p += TPR) top[0] = max_nan(top[0], piece_max<T, true>(row.load(z, p)));
        }
        row_join<true, TPR>(top, sm);
        fetch(r0 + step);  // (after the join: every thread has its pieces and entry)
        const float m = top[0], rtau = 1.0f / a.tau;
        const bool some = m > -INFINITY || isnan(m);
        const bool taught = top[1] > -INFINITY || isnan(top[1]);
        const bool soft = some && taught && a.alpha > 0.0f, hard = some && a.alpha < 1.0f && gold >= 0;
        const float k2 = kLog2e / a.tau;
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (soft)
            for (int j = t; j < k; j += TPR)
                if (ci[j] >= 0) {
                    const float l = (cw[j] - top[1]) * rtau, w = expf(l);
                    s[0] += w;
                    if (w > 0.0f)
                        s[1] += w * (l - (cz[j] - m) * rtau);  // (weight 0 on a class of -inf is 0)
                    else if (isnan(w))
                        s[1] = w;
                    cw[j] = w;
                }
        if (soft && hard)
            each([&](int, const float (&v)[E]) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float d = v[i] - m;
                    s[2] += exp2_hw(d * k2);
                    s[3] += exp2_hw(d * kLog2e);
                }
            });
        else if (soft || hard) {
            const float kk = soft ? k2 : kLog2e;
            float one = 0.0f;
            each([&](int, const float (&v)[E]) {
#pragma unroll
                for (int i = 0; i < E; ++i) one += exp2_hw((v[i] - m) * kk);
            });
            s[2] = soft ? one : 0.0f;
            s[3] = soft ? 0.0f : one;
        }
        row_join<false, TPR>(s, sm);
        const float ct = soft ? a.scale * a.alpha * a.tau : 0.0f, c1 = hard ? a.scale * (1.0f - a.alpha) : 0.0f;
        const float wt = soft ? ct / s[2] : 0.0f, w1 = hard ? c1 / s[3] : 0.0f;
        if (t == 0 && here && a.loss) {
            float loss = 0.0f;
            if (soft) loss = a.alpha * a.tau * a.tau * (s[1] / s[0] - logf(s[0]) + logf(s[2]));
            if (hard) loss += (1.0f - a.alpha) * (logf(s[3]) - (zgold - m));
            a.loss[r] = a.scale * loss;
        }
        if (!a.dz) {
            sync();  // the entries' arrays are the next row's
            continue;
        }
        // the entries' weights in the gradient; entry k is the gold class (read by all after the sync)
        for (int j = t; j < k; j += TPR)
            if (ci[j] >= 0) {
                if (soft)
                    cw[j] = ct * (cw[j] / s[0]);
                else
                    ci[j] = -1;
            }
        if (t == 0) {
            ci[a.k] = hard ? gold : -1;
            cw[a.k] = c1;
            cz[a.k] = zgold;
        }
        if (soft && hard)
            each([&](int p, const float (&v)[E]) {
                float g[E];
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float d = v[i] - m;
                    g[i] = fmaf(w1, exp2_hw(d * kLog2e), wt * exp2_hw(d * k2));
                }
                row.store_f32(a.dz, aligned, p, g);
            });
        else {
            const float kk = soft ? k2 : kLog2e, w = soft ? wt : w1;
            const bool any = soft || hard;
            each([&](int p, const float (&v)[E]) {
                float g[E];
#pragma unroll
                for (int i = 0; i < E; ++i) g[i] = any ? w * exp2_hw((v[i] - m) * kk) : 0.0f;
                row.store_f32(a.dz, aligned, p, g);
            });
        }
        sync();
        if (here)
            for (int j = t; j <= a.k; j += TPR) {
                const int c = ci[j];
                if (c < 0) continue;
                bool first = true;
                float w = cw[j];
                for (int i = 0; i <= a.k; ++i)
                    if (ci[i] == c) {
                        if (i < j) first = false;
                        if (i > j) w += cw[i];
                    }
                if (!first) continue;
                const float d = cz[j] - m;
                float g = 0.0f;
                if (soft) g = wt * exp2_hw(d * k2);
                if (hard) g = fmaf(w1, exp2_hw(d * kLog2e), g);
                a.dz[row.first() + c] = g - w;
            }
        sync();  // the entries' arrays are the next row's
    }
}

template <typename T, int TPR, int NP>
cudaError_t launch_rows(const stacklstm_op *op, const DistillArgs &a)
{
    constexpr int RPC = rows_per_cta(TPR);
    const size_t smem = (TPR > 32 ? (size_t)TPR * NP * 16 : 0) + (size_t)RPC * (a.k + 1) * 12;
    if (smem > 48 * 1024)
        if (cudaError_t e = smem_at_least((const void *)distill_rows<T, TPR, NP>, smem)) return e;
    // a CTA a row group, or as many CTAs as run at once where they read ahead
    const size_t groups = ceil_div(a.rows, RPC);
    const unsigned grid = (unsigned)(TPR > 32 && NP > 0 ? std::min(groups, (size_t)op->num_sms * row_ctas_per_sm(TPR)) : groups);
    distill_rows<T, TPR, NP><<<grid, row_cta(TPR), smem, op->stream>>>(a);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_distill(const stacklstm_op *op, const DistillArgs &a)
{
    int tpr, np;
    row_plan<T>(a.V, &tpr, &np);
#define SL_DIST(t, n) \
    if (tpr == t && np == n) return launch_rows<T, t, n>(op, a);
    SL_ROW_PLANS(SL_DIST)
#undef SL_DIST
    return cudaErrorInvalidValue;  // not reached
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
