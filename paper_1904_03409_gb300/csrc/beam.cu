// beam.cu -- beam search over StackLSTM hypotheses: the rows' normalisers, the selection over
// beams and classes, the reordering of the stacks and the push of a new state, and their C ABI
// (include/stacklstm.h, stacklstm_beam_*).
//
// Hypothesis k of sentence b has the score s[b][k] and the logits z[b][k][0 .. V); candidate
// (k, v) scores s[b][k] + (z[b][k][v] - lse[b][k]), each operation rounded to fp32, so that the
// order is a matter of the inputs alone. The K best of the K V candidates of a sentence go on,
// best first, of equal ones the lowest k V + v first. A candidate becomes one 64-bit key: the
// score's order in the upper half, the complement of its place in the lower one. Keys are
// distinct, and the K best are the same whatever order they are looked at in. Key 0 is no
// candidate (-inf or NaN).
#include "rowvec.cuh"

namespace sl {
namespace {

typedef unsigned long long u64;

constexpr int kSelThreads = 256;
constexpr int kSelItems = 32;                          // candidates a thread
constexpr int kSegment = kSelThreads * kSelItems;      // candidates a CTA
constexpr int kMergeItems = 16;                        // keys a thread and pass of the merge
constexpr int kMaxBeams = 64;

// ------------------------------------------------------------------ normalisers
template <typename T, int TPR, int NP>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR)
lse_rows(int rows, int V, const T *__restrict__ z, float *__restrict__ lse)
{
    constexpr int E = RowVec<T>::E, RPC = TPR == 32 ? 8 : 1;
    __shared__ float sm[kRowThreads / 32];
    const int r = blockIdx.x * RPC + (TPR == 32 ? threadIdx.x / 32 : 0), t = threadIdx.x % TPR;
    if (r >= rows) return;
    const RowVec<T> row(r, V, rows);
    const int n = row.pieces();
    float v[NP > 0 ? NP : 1][E];
    float m = -INFINITY, s = 0.0f;
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
    m = row_max<TPR>(m, sm);
    const float base = m == -INFINITY ? 0.0f : m;  // a row of -inf sums to 0: its lse is -inf
    auto add = [&](const float (&w)[E]) {
#pragma unroll
        for (int i = 0; i < E; ++i) s += exp2_hw((w[i] - base) * kLog2e);
    };
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
    s = row_sum<TPR>(s, sm);
    if (t == 0) lse[r] = base + logf(s);
}

template <typename T>
cudaError_t launch_lse(int rows, int V, const void *z, float *lse, cudaStream_t st)
{
    int tpr, np;
    row_plan<T>(V, &tpr, &np);
    const unsigned grid = ceil_div(rows, tpr == 32 ? 8 : 1);
#define SL_LSE(t, n) \
    if (tpr == t && np == n) lse_rows<T, t, n><<<grid, t == 32 ? 256 : t, 0, st>>>(rows, V, (const T *)z, lse);
    SL_LSE(32, 1) SL_LSE(32, 2) SL_LSE(32, 4)
    SL_LSE(kRowThreads, 0) SL_LSE(kRowThreads, 1) SL_LSE(kRowThreads, 2) SL_LSE(kRowThreads, 4)
    SL_LSE(kRowThreads, 8) SL_LSE(kRowThreads, 16)
#undef SL_LSE
    return cudaGetLastError();
}

// ------------------------------------------------------------------ selection
__device__ __forceinline__ u64 make_key(float score, uint32_t place)
{
    if (!(score > -INFINITY)) return 0;  // -inf and NaN
    const uint32_t b = __float_as_uint(score + 0.0f);  // -0 counts as 0
    const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return (u64)o << 32 | (0xFFFFFFFFu - place);
}
__device__ __forceinline__ float key_score(u64 key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}

struct SelShared {
    u64 top[kSelThreads];                // each thread's best key
    u64 best[kMaxBeams];                 // the K best, sorted
    u64 kth;
    int count, last;
    float score[kMaxBeams], lse[kMaxBeams];
    uint8_t done[kMaxBeams];
};

// The K best of the CTA's keys (PT a thread; list: room for K PT keys), sorted, into s.best.
// Each thread's best key is ranked among the threads': the K best keys are all in the K threads
// with the best of these, and none is below the K-th of them.
template <int PT>
__device__ __forceinline__ void block_topk(const u64 (&key)[PT], int K, SelShared &s, u64 *list)
{
    const int tid = threadIdx.x;
    u64 mine = 0;
#pragma unroll
    for (int i = 0; i < PT; ++i) mine = key[i] > mine ? key[i] : mine;
    __syncthreads();
    s.top[tid] = mine;
    if (tid == 0) {
        s.count = 0;
        s.kth = 1;  // fewer than K threads with a candidate: every one counts
    }
    if (tid < K) s.best[tid] = 0;
    __syncthreads();
    int rank = 0;
    if (mine)
        for (int i = 0; i < kSelThreads; ++i) rank += s.top[i] > mine;
    if (mine && rank == K - 1) s.kth = mine;
    __syncthreads();
    const u64 kth = s.kth;
    if (mine && rank < K) {
#pragma unroll
        for (int i = 0; i < PT; ++i)
            if (key[i] >= kth) list[atomicAdd(&s.count, 1)] = key[i];  // any order: they are ranked below
    }
    __syncthreads();
    const int n = s.count;
    for (int e = tid; e < n; e += kSelThreads) {
        const u64 k = list[e];
        int above = 0;
        for (int i = 0; i < n; ++i) above += list[i] > k;
        if (above < K) s.best[above] = k;
    }
    __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kSelThreads)
beam_select(int K, int V, int nseg, const T *__restrict__ z, const float *__restrict__ lse, const float *__restrict__ score,
            const uint8_t *__restrict__ done, u64 *__restrict__ part, int *__restrict__ arrived,
            float *__restrict__ out_score, int32_t *__restrict__ parent, int32_t *__restrict__ token)
{
    __shared__ SelShared s;
    extern __shared__ u64 list[];
    const int tid = threadIdx.x, b = blockIdx.y, seg = blockIdx.x;
    if (tid < K) {
        s.score[tid] = score[(size_t)b * K + tid];
        s.lse[tid] = lse ? lse[(size_t)b * K + tid] : 0.0f;
        s.done[tid] = done ? done[(size_t)b * K + tid] : 0;
    }
    __syncthreads();
    const uint32_t n = (uint32_t)K * (uint32_t)V;
    const T *zb = z + (size_t)b * n;
    {
        float v[kSelItems];
        const uint32_t e0 = (uint32_t)seg * kSegment + tid;
#pragma unroll
        for (int i = 0; i < kSelItems; ++i) {
            const uint32_t e = e0 + i * kSelThreads;
            v[i] = e < n ? to_f32(zb[e]) : -INFINITY;
        }
        u64 key[kSelItems];
#pragma unroll
        for (int i = 0; i < kSelItems; ++i) {
            const uint32_t e = e0 + i * kSelThreads;
            key[i] = 0;
            if (e < n) {
                const uint32_t k = e / (uint32_t)V;
                if (!s.done[k])
                    key[i] = make_key(__fadd_rn(s.score[k], __fsub_rn(v[i], s.lse[k])), e);
                else if (e == k * (uint32_t)V)
                    key[i] = make_key(s.score[k], e);
            }
        }
        block_topk<kSelItems>(key, K, s, list);
    }
    if (nseg > 1) {  // the sentence's last CTA joins the segments
        if (tid < K) part[((size_t)b * nseg + seg) * K + tid] = s.best[tid];
        __threadfence();
        __syncthreads();
        if (tid == 0) s.last = atomicAdd(&arrived[b], 1) == nseg - 1;
        __syncthreads();
        if (!s.last) return;
        __threadfence();
        if (tid == 0) arrived[b] = 0;  // for the next call
        const u64 *mine = part + (size_t)b * nseg * K;
        const int total = nseg * K, step = kSelThreads * (kMergeItems - 1);
        if (tid < K) s.best[tid] = 0;
        __syncthreads();
        for (int at = 0; at < total; at += step) {
            u64 key[kMergeItems];
#pragma unroll
            for (int i = 0; i < kMergeItems - 1; ++i) {
                const int e = at + i * kSelThreads + tid;
                key[i] = e < total ? __ldcg(mine + e) : 0;
            }
            key[kMergeItems - 1] = tid < K ? s.best[tid] : 0;  // the best so far
            block_topk<kMergeItems>(key, K, s, list);
        }
    }
    if (tid < K) {
        const u64 key = s.best[tid];
        const size_t o = (size_t)b * K + tid;
        if (!key) {
            out_score[o] = -INFINITY;
            parent[o] = token[o] = -1;
        } else {
            const uint32_t e = 0xFFFFFFFFu - (uint32_t)key, k = e / (uint32_t)V;
            out_score[o] = key_score(key);
            parent[o] = (int)k;
            token[o] = s.done[k] ? -1 : (int)(e - k * (uint32_t)V);
        }
    }
}

// ------------------------------------------------------------------ stacks
// The row of the old stacks that row n of the new ones comes from, and its pointer. A row whose
// candidate ran out (parent -1) keeps its own stack.
__device__ __forceinline__ int source_row(int n, int K, int S, const int32_t *parent, const int32_t *p, int *top, int32_t *err)
{
    const int b = n / K;
    int par = parent[n];
    if (par < -1 || par >= K) {
        atomicCAS(err, 0, (int)SL_ERR_ARG);
        par = -1;
    }
    const int src = par < 0 ? n : b * K + par;
    int at = p[src];
    if (at < 0 || at >= S) {
        atomicCAS(err, 0, (int)SL_ERR_ARG);
        at = min(max(at, 0), S - 1);
    }
    *top = at;
    return src;
}

// Row n (blockIdx.x) of the new stacks: the slots 0 .. p of its source row, and its top. PH and
// PC pieces (type Q) of h and c a slot; a CTA's threads take the pieces of its slots in order.
template <typename QH, typename QC>
__global__ void __launch_bounds__(256)
reorder_rows(int N, int K, int S, int PH, int PC, const int32_t *__restrict__ parent, const int32_t *__restrict__ p,
             const QH *__restrict__ h, const QC *__restrict__ c, int32_t *__restrict__ p_out, QH *__restrict__ h_out,
             QC *__restrict__ c_out, QH *__restrict__ top_h, QC *__restrict__ top_c, int32_t *err)
{
    const int n = blockIdx.x;
    int top;
    const int src = source_row(n, K, S, parent, p, &top, err);
    const int per = PH + PC;
    for (int s = blockIdx.y; s <= top; s += gridDim.y) {
        const size_t from = (size_t)s * N + src, to = (size_t)s * N + n;
        for (int i = threadIdx.x; i < per; i += blockDim.x) {
            if (i < PH) {
                const QH v = h[from * PH + i];
                h_out[to * PH + i] = v;
                if (s == top && top_h) top_h[(size_t)n * PH + i] = v;
            } else {
                const QC v = c[from * PC + i - PH];
                c_out[to * PC + i - PH] = v;
                if (s == top && top_c) top_c[(size_t)n * PC + i - PH] = v;
            }
        }
    }
    if (blockIdx.y == 0 && threadIdx.x == 0) p_out[n] = top;
}

// Row n: the new state into slot p + 1 of a push, p moved by the op, the new top out.
template <typename QH, typename QC>
__global__ void __launch_bounds__(128)
push_rows(int N, int S, int PH, int PC, const int8_t *__restrict__ ops, const QH *__restrict__ h_new,
          const QC *__restrict__ c_new, int32_t *__restrict__ p, QH *__restrict__ h, QC *__restrict__ c,
          QH *__restrict__ top_h, QC *__restrict__ top_c, int32_t *err)
{
    const int n = blockIdx.x;
    int at = p[n], op = ops[n];
    if (threadIdx.x == 0) {
        if (at < 0 || at >= S) atomicCAS(err, 0, (int)SL_ERR_ARG);
        if (op < -1 || op > 1) atomicCAS(err, 0, (int)SL_ERR_OP);
        else if (op == -1 && at <= 0) atomicCAS(err, 0, (int)SL_ERR_UNDERFLOW);
        else if (op == 1 && at >= S - 1) atomicCAS(err, 0, (int)SL_ERR_ARG);
    }
    at = min(max(at, 0), S - 1);
    if (op < -1 || op > 1 || at + op < 0 || at + op >= S) op = 0;  // as a hold
    const int to = at + op;
    for (int i = threadIdx.x; i < PH + PC; i += blockDim.x) {
        const size_t slot = (size_t)to * N + n;
        if (i < PH) {
            QH v;
            if (op == 1) {
                v = h_new[(size_t)n * PH + i];
                h[slot * PH + i] = v;
            } else {
                v = h[slot * PH + i];
            }
            if (top_h) top_h[(size_t)n * PH + i] = v;
        } else {
            const int j = i - PH;
            QC v;
            if (op == 1) {
                v = c_new[(size_t)n * PC + j];
                c[slot * PC + j] = v;
            } else {
                v = c[slot * PC + j];
            }
            if (top_c) top_c[(size_t)n * PC + j] = v;
        }
    }
    __syncthreads();  // every thread has read p
    if (threadIdx.x == 0) p[n] = to;
}

}  // namespace
}  // namespace sl

using namespace sl;

extern "C" {

sl_status stacklstm_beam_create(stacklstm_op_t *out, int B, int K, int V, int S, int H, sl_dtype dtype, int device,
                                void *stream)
{
    if (!out) return SL_ERR_ARG;
    *out = nullptr;
    if (B < 1 || K < 1 || V < 1 || S < 1 || H < 1 || (dtype != SL_FP32 && dtype != SL_BF16)) return SL_ERR_ARG;
    if (K > kMaxBeams || B > 65535 || (long long)K * V > (1LL << 30) || H > (1 << 24)) return SL_ERR_UNSUPPORTED;
    sl_status st;
    stacklstm_op *op = op_new(SL_OP_BEAM, dtype, device, stream, &st);
    if (!op) return st;
    op->R = B * K; op->B = B; op->beams = K; op->V = V; op->S = S; op->H = H;
    OpDevice guard(device);
    const size_t nseg = ceil_div((size_t)K * V, kSegment);
    cudaError_t e = op_workspace(op, 0, (size_t)B * nseg * K * 8);
    if (!e) e = op_workspace(op, 1, (size_t)B * 4);
    if (!e) e = cudaMemset(op->ws[1], 0, (size_t)B * 4);
    if (!e) e = smem_at_least((const void *)beam_select<float>, (size_t)kMaxBeams * kSelItems * 8);
    if (!e) e = smem_at_least((const void *)beam_select<__nv_bfloat16>, (size_t)kMaxBeams * kSelItems * 8);
    if (e) {
        stacklstm_op_destroy(op);
        return SL_ERR_OOM;
    }
    *out = op;
    return SL_OK;
}

sl_status stacklstm_beam_lse(stacklstm_op_t op, const void *logits, float *lse)
{
    if (!op || op->kind != SL_OP_BEAM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_pointers({logits, lse}, {})) return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    const cudaError_t e = op->dt == SL_BF16 ? launch_lse<__nv_bfloat16>(op->R, op->V, logits, lse, op->stream)
                                            : launch_lse<float>(op->R, op->V, logits, lse, op->stream);
    return e ? op_cuda(op, e, "stacklstm_beam_lse") : SL_OK;
}

sl_status stacklstm_beam_select(stacklstm_op_t op, const void *logits, const float *lse, const float *score,
                                const uint8_t *done, float *new_score, int32_t *parent, int32_t *token)
{
    if (!op || op->kind != SL_OP_BEAM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_pointers({logits, score, new_score, parent, token}, {lse, done}))
        return op_fail(op, SL_ERR_ARG, m);
    if (new_score == score) return op_fail(op, SL_ERR_ARG, "new_score must not be score: it is read by the whole sentence");
    OpDevice guard(op->device);
    const int K = op->beams, V = op->V, nseg = (int)ceil_div((size_t)K * V, kSegment);
    const dim3 grid(nseg, op->B);
    const size_t smem = (size_t)K * kSelItems * 8;
    if (op->dt == SL_BF16)
        beam_select<<<grid, kSelThreads, smem, op->stream>>>(K, V, nseg, (const __nv_bfloat16 *)logits, lse, score, done,
                                                             (u64 *)op->ws[0], (int *)op->ws[1], new_score, parent, token);
    else
        beam_select<<<grid, kSelThreads, smem, op->stream>>>(K, V, nseg, (const float *)logits, lse, score, done,
                                                             (u64 *)op->ws[0], (int *)op->ws[1], new_score, parent, token);
    const cudaError_t e = cudaGetLastError();
    return e ? op_cuda(op, e, "stacklstm_beam_select") : SL_OK;
}

sl_status stacklstm_beam_reorder(stacklstm_op_t op, const int32_t *parent, const int32_t *p, const void *h_stack,
                                 const float *c_stack, int32_t *p_out, void *h_out, float *c_out, void *top_h, float *top_c)
{
    if (!op || op->kind != SL_OP_BEAM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_pointers({parent, p, h_stack, c_stack, p_out, h_out, c_out}, {top_h, top_c}))
        return op_fail(op, SL_ERR_ARG, m);
    if (p_out == p || h_out == h_stack || c_out == c_stack)
        return op_fail(op, SL_ERR_ARG, "the new stacks must not be the old ones: rows are read after others are written");
    OpDevice guard(op->device);
    const int N = op->R, K = op->beams, S = op->S, H = op->H;
    const bool bf = op->dt == SL_BF16;
    const dim3 grid(N, std::min(S, 64));
    if (H % 8 == 0)
        reorder_rows<<<grid, 256, 0, op->stream>>>(N, K, S, H / (bf ? 8 : 4), H / 4, parent, p, (const uint4 *)h_stack,
                                                   (const uint4 *)c_stack, p_out, (uint4 *)h_out, (uint4 *)c_out,
                                                   (uint4 *)top_h, (uint4 *)top_c, op->err);
    else if (bf)
        reorder_rows<<<grid, 256, 0, op->stream>>>(N, K, S, H, H, parent, p, (const uint16_t *)h_stack,
                                                   (const uint32_t *)c_stack, p_out, (uint16_t *)h_out, (uint32_t *)c_out,
                                                   (uint16_t *)top_h, (uint32_t *)top_c, op->err);
    else
        reorder_rows<<<grid, 256, 0, op->stream>>>(N, K, S, H, H, parent, p, (const uint32_t *)h_stack,
                                                   (const uint32_t *)c_stack, p_out, (uint32_t *)h_out, (uint32_t *)c_out,
                                                   (uint32_t *)top_h, (uint32_t *)top_c, op->err);
    const cudaError_t e = cudaGetLastError();
    return e ? op_cuda(op, e, "stacklstm_beam_reorder") : SL_OK;
}

sl_status stacklstm_beam_push(stacklstm_op_t op, const int8_t *ops, const void *h_new, const float *c_new, int32_t *p,
                              void *h_stack, float *c_stack, void *top_h, float *top_c)
{
    if (!op || op->kind != SL_OP_BEAM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_pointers({ops, h_new, c_new, p, h_stack, c_stack}, {top_h, top_c}))
        return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    const int N = op->R, S = op->S, H = op->H;
    const bool bf = op->dt == SL_BF16;
    if (H % 8 == 0)
        push_rows<<<N, 128, 0, op->stream>>>(N, S, H / (bf ? 8 : 4), H / 4, ops, (const uint4 *)h_new, (const uint4 *)c_new,
                                             p, (uint4 *)h_stack, (uint4 *)c_stack, (uint4 *)top_h, (uint4 *)top_c, op->err);
    else if (bf)
        push_rows<<<N, 128, 0, op->stream>>>(N, S, H, H, ops, (const uint16_t *)h_new, (const uint32_t *)c_new, p,
                                             (uint16_t *)h_stack, (uint32_t *)c_stack, (uint16_t *)top_h,
                                             (uint32_t *)top_c, op->err);
    else
        push_rows<<<N, 128, 0, op->stream>>>(N, S, H, H, ops, (const uint32_t *)h_new, (const uint32_t *)c_new, p,
                                             (uint32_t *)h_stack, (uint32_t *)c_stack, (uint32_t *)top_h,
                                             (uint32_t *)top_c, op->err);
    const cudaError_t e = cudaGetLastError();
    return e ? op_cuda(op, e, "stacklstm_beam_push") : SL_OK;
}

}  // extern "C"
